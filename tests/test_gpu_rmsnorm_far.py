"""The norm where single steps of the formula leave fp32's range and its results
do not: weights whose |y| passes it and whose scale, |y| / 127, does not; an eps
near its end.  Tolerances: test_gpu_rmsnorm."""
import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn
from test_gpu_rmsnorm import R, TYPES

pytestmark = pytest.mark.gpu
MOST = torch.finfo(torch.float32).max


def _check(x, weight, eps):
    _, y, q, scale = bnn.bnn_rmsnorm(x.cuda(), weight.cuda(), None, eps, want_y=True)
    _, yr, qr, sr = ref.rmsnorm(x, weight, None, eps)
    assert torch.equal(q.cpu(), qr)
    assert torch.isfinite(sr).all() and (sr < MOST).all()
    torch.testing.assert_close(scale.cpu().double(), sr, rtol=R, atol=1e-44)
    half, most = torch.finfo(x.dtype).eps / 2, torch.finfo(x.dtype).max
    inside = yr.abs() <= most * (1 - 2 * half)
    torch.testing.assert_close(y.cpu().double()[inside], yr[inside], rtol=R + half,
                               atol=torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps)
    beyond = yr.abs() > most * (1 + 2 * half)
    assert torch.isinf(y.cpu()[beyond]).all()
    return beyond


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 1000, 5000, 40000])
def test_largest_beyond_the_range(kind, D):
    """One loud value under a weight near the type's largest: |y| up to sqrt(D) of it."""
    g = torch.Generator().manual_seed(D)
    x = 1e-12 * torch.randn(6, D, generator=g)
    x[torch.arange(6), torch.randint(0, D, (6,), generator=g)] = torch.tensor([1e-10, -1e-10, 1e-3, -2.0, 1e-10, 1e-8])
    weight = 1e37 * (1 + torch.rand(D, generator=g))
    weight[x[0].abs().argmax()] = 3e38
    x[2:4] *= 1e-7  # (so that h w stays within fp32 for every row)
    beyond = _check(x.to(TYPES[kind]), weight.to(TYPES[kind]), 1e-30)
    assert beyond.any()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("eps", [MOST, 3.4e38, 1e37, 1e36])
def test_large_eps(kind, eps):
    g = torch.Generator().manual_seed(7)
    for D in (8, 700, 3000):
        x = 3e17 * (1 + torch.rand(4, D, generator=g))
        _check((x * (2.0 / D ** 0.5)).to(TYPES[kind]), torch.randn(D, generator=g).to(TYPES[kind]), eps)
