"""Log probabilities of int32 logits that fp32 does not tell apart: sums beyond
2^24, whose small differences decide.

Tolerances are test_gpu_logprobs', and for c v in 64 bits, where v has up to 31
bits and c 24, two roundings of 2^-53 |c v|: 2^-51 |z| covers them in ln p (an
answer's and the reference's), twice that in the entropy (two parts' references
lie off against each other, and each part's weight and mean move)."""
import math

import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn
from test_gpu_logprobs import _near

pytestmark = pytest.mark.gpu


def _check(z, ids, top_k, scale):
    got = bnn.bnn_logprobs(z.cuda(), ids.cuda(), top_k, scale)
    torch.cuda.synchronize()
    given, entropy, top_ids, top = ref.logprobs(z, ids, top_k, scale)
    V = z.shape[1]
    far = z.abs().max().item() * scale
    Z = max(-v[torch.isfinite(v)].min().item() for v in (given, top))
    assert torch.equal(got[2].cpu(), top_ids)
    for a, b in ((got[0], given), (got[3], top)):
        _near(a, b, 2.0 ** -24 * (3 * Z + V / 512 + 200) + 2.0 ** -51 * far)
        assert (a <= 0).all()
    _near(got[1], entropy, 2.0 ** -24 * (V / 512 + 200) * (3 + math.log(V)) + 2.0 ** -50 * far)


NEAR = [[2 ** 30 + 60, 2 ** 30 + 10], [2 ** 25 + 1, 2 ** 25 - 4, 2 ** 25 + 3], [-2 ** 30 - 1, -2 ** 30 - 2, -2 ** 30],
        [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 9], [-2 ** 31 + 7, -2 ** 31 + 6, -2 ** 31 + 7], [2 ** 24 + 1, 2 ** 24, 2 ** 24 + 3],
        [-2 ** 24 - 1, -2 ** 24 - 2, -2 ** 24 - 4], [5, 3, 4]]


@pytest.mark.parametrize("scale", [1.0, 0.25, 3.0])
@pytest.mark.parametrize("values", NEAR)
def test_few_answers(values, scale):
    """Nothing else in the row: the probabilities add up to 1."""
    z = torch.tensor([values, values[::-1]], dtype=torch.int32)
    n = len(values)
    ids = torch.arange(n, dtype=torch.int32).repeat(2, 1)
    _check(z, ids, n, scale)
    lp = bnn.bnn_logprobs(z.cuda(), ids.cuda(), logit_scale=scale)[0].cpu().double()
    assert ((torch.exp(lp).sum(1) - 1).abs() <= 2.0 ** -16).all()


@pytest.mark.parametrize("T, V", [(len(NEAR), 900), (len(NEAR), 5000), (1, 70000), (len(NEAR), 40001), (176, 17000), (600, 17001)])
@pytest.mark.parametrize("scale", [1.0, 3.0])
def test_among_many(T, V, scale):
    """The rest out of the way, in another part of the row or beside them."""
    g = torch.Generator().manual_seed(V)
    z = torch.full((T, V), -2 ** 31, dtype=torch.int32)
    ids = torch.empty(T, 2, dtype=torch.int32)
    for t in range(T):
        values = NEAR[t % len(NEAR)]
        at = torch.randperm(V, generator=g)[:len(values)]
        z[t, at] = torch.tensor(values, dtype=torch.int32)
        ids[t] = at[:2]
    _check(z, ids, 2, scale)


@pytest.mark.parametrize("T, V", [(5, 800), (3, 8192), (4, 30003), (165, 16400)])
@pytest.mark.parametrize("scale", [1.0, 0.125, 2.0 ** -12, 2.0 ** -31])
def test_dense_rows(T, V, scale):
    """Every value within 40 steps of the scale of a far one."""
    g = torch.Generator().manual_seed(V + 1)
    wide = min(int(40 / scale), 2 ** 30)
    base = torch.tensor([2 ** 25, 2 ** 30, -2 ** 30, 2 ** 31 - 1 - wide, -2 ** 31], dtype=torch.int64)
    z = base[torch.arange(T) % 5][:, None] + torch.randint(0, wide + 1, (T, V), generator=g)
    z = z.clamp(-2 ** 31, 2 ** 31 - 1).to(torch.int32)
    _check(z, torch.randint(0, V, (T, 3), generator=g, dtype=torch.int32), 9, scale)
