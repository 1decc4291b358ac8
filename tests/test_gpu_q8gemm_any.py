"""8-bit matrix product of rows that lie anywhere, on both of its tiles: K shorter
than 16, than a step of 128, of whole steps and not, rows and outputs that end
inside a tile, each output type, bit by bit.  Which size takes which tile:
test_q8_any_plans."""
import pytest

from test_gpu_q8gemm import _check, pytestmark  # noqa: F401

# (M, N, K); the first four on tiles of 128
LARGE = [(2050, 2060), (16385, 130), (129, 16300), (2048, 2048)]
SMALL = [(700, 900), (65, 3000), (1, 9000), (2000, 63)]
KS = [7, 15, 16, 33, 128, 129, 1001, 1024, 2175]


@pytest.mark.parametrize("M, N", LARGE + SMALL)
@pytest.mark.parametrize("K", KS)
def test_tiles(M, N, K):
    """x's rows on odd bytes, w's on 16-byte ones with a distance of their own."""
    if M <= 16 and K >= 16:
        K += 8192  # (few rows of less are the other kernel's)
    kind = ("fp32", "fp16", "bf16")[(K + N) % 3]
    _check(M, N, K, kind, x_at=(K + 1, 3), w_at=(K + 5, 0))


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M, N", [(2050, 2060), (300, 333)])
def test_types_and_options(M, N, kind):
    for K in (15, 1001):
        _check(M, N, K, kind, x_at=(K, 0), w_at=(K, 1))
        _check(M, N, K, kind, scales=False, bias=False, x_at=(K, 1), w_at=(K, 0))
    # aligned but for the weights' start, their distance, x's distance
    _check(M, N, 1024, kind, w_at=(1024, 8))
    _check(M, N, 1024, kind, bias=False, w_at=(1032, 0))
    _check(M, N, 1024, kind, scales=False, x_at=(1025, 0))


@pytest.mark.parametrize("M, N, K", [(1, 70, 10001), (1, 4100, 8209), (300, 1, 1001), (2000, 1, 15), (1, 1, 20000)])
def test_one_row(M, N, K):
    """A single row whose distance is odd, on a 16-byte step and off it, with
    nothing of its buffer behind it."""
    pad = (K + 15) // 16 * 16
    for first in (0, 16, 5):
        _check(M, N, K, x_at=(K if M == 1 else pad, first if M == 1 else 0), w_at=(K if N == 1 else pad, first if N == 1 else 0))
