"""8-bit matrix product against its definition (quant_ref).  The sums are exact
and the steps after them are stated one by one in fp32, so every output is asked
for bit by bit."""
import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _bytes(g, M, K):
    return torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int8)


def _laid(t, stride, first=0, junk=-128):
    """t's rows on the GPU, `stride` bytes apart from byte `first` on, with junk
    between them, and nothing of the buffer behind the last one."""
    M, K = t.shape
    flat = torch.full((first + (M - 1) * stride + K,), junk, dtype=torch.int8)
    flat[first:].as_strided((M, K), (stride, 1)).copy_(t)
    return flat.cuda()[first:].as_strided((M, K), (stride, 1))


def _operands(g, M, N, K):
    return (_bytes(g, M, K), _bytes(g, N, K), torch.rand(M, generator=g) / 64 + 1e-3,
            torch.rand(N, generator=g) / 64 + 1e-3, torch.randn(N, generator=g))


def _check(M, N, K, kind="fp32", scales=True, bias=True, x_at=None, w_at=None, seed=0):
    g = torch.Generator().manual_seed(M + 131 * N + 7919 * K + seed)
    x, w, xs, ws, b = _operands(g, M, N, K)
    if not scales:
        xs = ws = None
    b = b if bias else None
    pad = (K + 15) // 16 * 16
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    y = bnn.bnn_q8gemm(_laid(x, *(x_at or (pad, 0))), _laid(w, *(w_at or (pad, 0))), dev(xs), dev(ws), dev(b),
                       dtype=TYPES[kind])
    torch.cuda.synchronize()
    want = ref.q8gemm(x, w, xs, ws, b, TYPES[kind])
    assert y.shape == (M, N) and torch.equal(y.cpu(), want)


SIZES = [(1, 1, 1), (1, 5, 3), (1, 16, 64), (1, 33, 100), (1, 4096, 4096), (1, 1000, 4097), (2, 40, 16),
         (3, 257, 129), (7, 2050, 1100), (8, 4096, 512), (16, 100, 8192), (17, 300, 700), (31, 64, 4096),
         (32, 1024, 1024), (33, 65, 4111), (63, 129, 255), (64, 512, 640), (65, 64, 127), (100, 100, 128),
         (128, 128, 256), (129, 257, 130), (200, 1030, 2050), (256, 4096, 4096), (777, 2050, 1100),
         (513, 511, 1029), (1024, 1024, 1024), (2050, 300, 96), (300, 4100, 17), (1500, 1500, 512),
         # tiles of 128 (one and two per CU) and 256, K shorter than a stage, of
         # whole stages, and short last ones with whole chunks and without
         (1000, 4100, 100), (2000, 2000, 16), (1100, 3900, 1024), (1030, 3700, 1104), (2000, 4200, 31),
         (2000, 4100, 384), (2100, 4000, 400), (4100, 3900, 16), (3900, 4100, 256), (3850, 4000, 1029),
         (4096, 4096, 640), (4000, 4001, 99), (300, 300, 400), (1050, 4000, 1029),
         (1000, 4000, 100), (1000, 4000, 1024), (1000, 4001, 400), (990, 4000, 1029),
         (2000, 4000, 31), (2000, 4001, 384), (2000, 4000, 400), (1950, 3999, 1029), (4000, 4001, 400),
         # few rows of more than x's registers hold
         (1, 70, 10000), (16, 100, 8208), (5, 64, 20011), (40, 70, 4112), (20, 4096, 4096)]


@pytest.mark.parametrize("M, N, K", SIZES)
def test_sizes(M, N, K):
    _check(M, N, K)
    _check(M, N, K, "bf16", bias=False)


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M, N, K", [(1, 300, 200), (20, 300, 1000), (70, 300, 200), (300, 333, 444)])
def test_types_and_options(M, N, K, kind):
    _check(M, N, K, kind, scales=False, bias=False)
    _check(M, N, K, kind, scales=False)
    _check(M, N, K, kind, bias=False)


@pytest.mark.parametrize("M", [1, 9, 40, 130, 700])
@pytest.mark.parametrize("x_at, w_at", [((0, 0), (0, 0)), ((0, 1), (0, 3)), ((5, 7), (16, 0)), ((16, 0), (3, 2)),
                                        ((64, 0), (4096, 0))])
def test_rows_anywhere(M, x_at, w_at):
    for K in (15, 16, 17, 144, 1001, 1024):
        pad = (K + 15) // 16 * 16
        at = lambda a: ((pad if a[0] % 16 == 0 and a[0] else K) + a[0], a[1])  # noqa: E731
        _check(M, 200, K, x_at=at(x_at), w_at=at(w_at))


@pytest.mark.parametrize("M", [1, 30, 200])
def test_largest_sums(M):
    """K at its limit with every product 2^14: sums up to 2^31 - 2^14."""
    K, N = 131071, 70
    x, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    w[1] = 127
    y = bnn.bnn_q8gemm(_laid(x, K), _laid(w, K))
    want = torch.full((M, N), float(K * 16384))
    want[:, 1] = float(-K * 128 * 127)
    assert torch.equal(y.cpu(), want.to(torch.float32))


@pytest.mark.parametrize("M", [1, 50, 300])
def test_buffers_beyond_4_gib(M):
    """Weight rows far apart: offsets that pass 32 bits."""
    K, N, stride = 64, 70, 1 << 26
    g = torch.Generator().manual_seed(3)
    x, w, xs, ws, _ = _operands(g, M, N, K)
    flat = torch.zeros((N - 1) * stride + K, dtype=torch.int8, device="cuda")
    far = flat.as_strided((N, K), (stride, 1))
    far.copy_(w)
    y = bnn.bnn_q8gemm(x.cuda(), far, xs.cuda(), ws.cuda())
    assert torch.equal(y.cpu(), ref.q8gemm(x, w, xs, ws))


def test_outputs_stay_inside():
    """Nothing is written beside y, and a caller's y is the one returned."""
    g = torch.Generator().manual_seed(4)
    for M, N, K in ((1, 30, 64), (40, 70, 96), (130, 200, 300)):
        x, w, xs, ws, b = _operands(g, M, N, K)
        store = torch.full((M * N + 64,), 7.0, device="cuda")
        out = store[32:32 + M * N].view(M, N)
        assert bnn.bnn_q8gemm(x.cuda(), w.cuda(), xs.cuda(), ws.cuda(), b.cuda(), out=out) is out
        assert torch.equal(out.cpu(), ref.q8gemm(x, w, xs, ws, b))
        assert (store[:32] == 7).all() and (store[32 + M * N:] == 7).all()
    assert bnn.bnn_q8gemm(x.cuda()[:0], w.cuda()).shape == (0, 200)
