"""Sizes of the workspaces of the mixture-of-experts calls (CPU only): a buffer
for the most rows that a program passes is enough for any fewer, and holds what
the kernels put there."""
import ctypes

import pytest

import test_expert_plans as plans
from paper_1808_00209_amd import bnn


def _sizes(call, make, rows):
    n, out = ctypes.c_size_t(), []
    for M in rows:
        assert call(*make(M), ctypes.byref(n)) == bnn.BNN_OK
        out.append(n.value)
    return out


def _never_falls(sizes, rows):
    for a, b, m in zip(sizes, sizes[1:], rows[1:]):
        assert b >= a, "at %d rows" % m


LORA_ROWS = list(range(0, 17000)) + list(range(17000, 70000, 37))


@pytest.mark.parametrize("K", [1, 1000, 1025, 4096, 65536])
@pytest.mark.parametrize("rank", [8, 16, 64, 72, 256])
def test_bgemm_lora(rank, K):
    lib = bnn.load()
    make = lambda M: (ctypes.byref(bnn.LoraDesc(M, 64, K, 3, rank, 2, 2)),)  # noqa: E731
    sizes = _sizes(lib.bnn_bgemm_lora_workspace_size, make, LORA_ROWS)
    _never_falls(sizes, LORA_ROWS)
    for M, n in list(zip(LORA_ROWS, sizes))[::97]:
        slices = plans._call("down_slices", M, K, rank) if M else 0
        assert n >= M * (slices * rank + bnn.words(K)) * 4  # u and sign bits
        assert n <= (M * (rank + bnn.words(K)) + 8160 * rank) * 4


GROUP_ROWS = list(range(16000, 40000)) + list(range(40000, 1 << 24, 4099)) + [(1 << 24) - 1]
GROUP_ROWS += [m for k in range(2, 65) for m in (k * 262144 - 1, k * 262144 + 1) if m < 1 << 24]


@pytest.mark.parametrize("G", [1, 256, 1024])
def test_group_rows(G):
    rows = sorted(GROUP_ROWS)
    sizes = _sizes(bnn.load().bnn_group_rows_workspace_size, lambda M: (M, G), rows)
    _never_falls(sizes, rows)
    for M, n in zip(rows, sizes):
        if M > 16384:  # a count per chunk of at least 2048 rows and group
            steps = (M + 2047) // 2048
            chunk = 2048 * ((steps + 127) // 128)
            assert n >= (M + chunk - 1) // chunk * (G + 1) * 4


@pytest.mark.parametrize("N, K", [(1, 1), (700, 1000), (4096, 4096), (65536, 65535)])
def test_experts_sum(N, K):
    most = min(1 << 16, (1 << 28) // (4 * ((N + 63) // 64)))
    rows = list(range(0, min(most, 9000))) + list(range(9000, most, 101))
    make = lambda T: (ctypes.byref(bnn.ExpertsDesc(T, 4, 8, N, K, 0)),)  # noqa: E731
    sizes = _sizes(bnn.load().bnn_experts_sum_workspace_size, make, rows)
    _never_falls(sizes, rows)
