"""The 8-bit layers and the log probabilities at the ends of what a call accepts:
the most rows, the most outputs, outputs and rows whose offsets pass 32 bits.
The product's outputs are exact here (sums below 2^24, no scales), and looked at
where an offset would wrap and at both ends; uniform rows have ln p -ln V."""
import math

import pytest
import torch

from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu
MOST = (1 << 24) - 1  # rows


def _bytes(g, M, K, stride):
    rows = torch.empty(M * stride, dtype=torch.int8, device="cuda").random_(-128, 128, generator=g)
    return rows.as_strided((M, K), (stride, 1))


def _same(y, x, w):
    """y's rows against exact products, some hundred at a time."""
    M, N = y.shape
    last = [0, M - 200] + [max(0, min(M - 200, at // N - 100)) for at in (1 << 30, 1 << 31, 1 << 32)]
    wd = w.double()
    for m in sorted(set(max(0, v) for v in last)):
        part = slice(m, min(m + 200, M))
        assert torch.equal(y[part].double(), x[part].double() @ wd.T), m


@pytest.mark.parametrize("M, N, K, stride, dtype", [
    ((1 << 21) + 5, 2050, 32, 32, torch.float16),    # tiles of 256, more than 2^32 outputs
    ((1 << 21) + 5, 2050, 33, 33, torch.float32),    # rows that lie anywhere
    (MOST, 1, 16, 16, torch.float32), (MOST, 33, 20, 32, torch.float32), (MOST, 3, 7, 7, torch.float32),
    (1, 1 << 20, 64, 64, torch.float32), (16, 1 << 20, 100, 100, torch.float32), (40, 1 << 20, 100, 112, torch.float32)])
def test_products(M, N, K, stride, dtype):
    g = torch.Generator(device="cuda").manual_seed(N + K)
    x, w = _bytes(g, M, K, stride), _bytes(g, N, K, stride)
    if dtype is torch.float16:  # (sums that fp16 holds)
        x.remainder_(4)
        w.remainder_(8)
    y = bnn.bnn_q8gemm(x, w, dtype=dtype)
    _same(y, x, w)


@pytest.mark.parametrize("V, dtype", [(3, torch.float32), (1025, torch.bfloat16)])
def test_most_rows_of_answers(V, dtype):
    z = torch.zeros(MOST, V, dtype=dtype, device="cuda")
    rows = torch.tensor([0, 1, (1 << 21) + 3, 4190209, 1 << 23, MOST - 1], device="cuda")
    z[rows, 2] = 4.0  # (4190209 * 1025: beyond 2^32)
    ids = torch.full((MOST,), 2, dtype=torch.int32, device="cuda")
    logp, entropy, top_ids, top = bnn.bnn_logprobs(z, ids, 1)
    tol = 2.0 ** -24 * (3 * 12 + 210)
    want = 4 - math.log(math.exp(4) + V - 1)
    assert ((logp[rows].double() - want).abs() <= tol).all() and (top_ids[rows] == 2).all()
    assert torch.equal(top[rows, 0], logp[rows])
    logp[rows], top[rows], top_ids[rows], entropy[rows] = -math.log(V), -math.log(V), 0, math.log(V)
    assert ((logp + math.log(V)).abs() <= tol).all() and ((top + math.log(V)).abs() <= tol).all()
    assert (top_ids == 0).all() and ((entropy - math.log(V)).abs() <= 210 * 2.0 ** -24 * (3 + math.log(V))).all()


def test_most_rows_of_the_norm():
    """Rows of one value: q is 127 of its sign, y the sign itself."""
    x = torch.empty(MOST, 1, dtype=torch.bfloat16, device="cuda")
    x.copy_((torch.arange(MOST, device="cuda")[:, None] % 7 - 3).bfloat16())
    _, y, q, scale = bnn.bnn_rmsnorm(x, eps=0.0, want_y=True)
    sign = torch.sign(x.float())
    assert torch.equal(q.float(), 127 * sign) and torch.equal(y.float(), sign)
    assert ((scale - sign[:, 0].abs() / 127).abs() <= 2.0 ** -22 / 127).all()
