"""Log probabilities on every form of the kernel: one, four and sixteen waves per
row, rows in parts (also more parts than a wave has lanes), with ends inside a
step and a group of 8, waves and parts that get nothing.  Which size takes which
form: test_logprobs_plans.  Tolerances: test_gpu_logprobs."""
import math

import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn
from test_gpu_logprobs import TYPES, _logits, _near

pytestmark = pytest.mark.gpu

# 16 waves; four on whole rows; parts (300001 and more: over 64 of them); one wave
SIZES = [(161, 16384), (301, 20003), (511, 17000), (160, 33000), (513, 16385), (180, 9001), (2, 8193), (1, 300001), (3, 1 << 20),
         (159, 12289), (30, 100000), (2048, 4096), (2049, 1023), (7, 1024), (1, 1 << 24)]


def _compare(z, ids, scale, ks=(0, 1, 8, 32)):
    """Every number of alternatives against one reference with the most of them."""
    V = z.shape[1]
    dev, at = z.cuda(), ids.cuda()
    given, entropy, top_ids, top = ref.logprobs(z, ids, min(max(ks), V), scale)
    Z = max([-v[torch.isfinite(v)].min().item() for v in (given, top) if torch.isfinite(v).any()] + [0.0])
    for k in ks:
        got = bnn.bnn_logprobs(dev, at, min(k, V), scale)
        _near(got[0], given, 2.0 ** -24 * (3 * Z + V / 512 + 200))
        _near(got[1], entropy, 2.0 ** -24 * (V / 512 + 200) * (3 + math.log(V)))
        if k:
            assert torch.equal(got[2].cpu(), top_ids[:, :k])
            _near(got[3], top[:, :k], 2.0 ** -24 * (3 * Z + V / 512 + 200))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("T, V", SIZES)
def test_forms(T, V, kind):
    g = torch.Generator().manual_seed(V + T)
    ids = torch.randint(0, V, (T, 2), generator=g, dtype=torch.int32)
    _compare(_logits(g, T, V, kind), ids, 1 / 16 if kind == "int32" else 1.0)


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T, V", [(176, 20003), (600, 9000), (10, 300001)])
def test_masks(T, V, kind):
    """Rows out of reach but for a few answers or altogether, NaN, infinities,
    equal values and the lowest one, each beside ordinary rows."""
    g = torch.Generator().manual_seed(V)
    z = _logits(g, T, V, kind)
    low = torch.finfo(TYPES[kind]).min
    for t in range(T):
        case = t % 10
        if case == 0:
            z[t][torch.rand(V, generator=g) < 0.999] = -math.inf
        elif case == 1:
            z[t] = -math.inf
        elif case == 2:
            z[t, V // 3] = math.nan
        elif case == 3:
            z[t, V - 1] = math.inf
        elif case == 4:
            z[t] = 1.5
        elif case == 5:
            z[t] = low
        elif case == 6:
            z[t, : V - 3] = -math.inf
        elif case == 7:
            z[t, 5:] = -math.inf
        elif case == 8:
            z[t, ::2] = z[t].max()
    ids = torch.randint(-1, V + 1, (T, 3), generator=g, dtype=torch.int32)
    _compare(z, ids, 1.0, (0, 20))


def test_integers_equal_and_rising():
    g = torch.Generator().manual_seed(5)
    for T, V in ((165, 16400), (4, 300001)):
        z = torch.randint(-3, 4, (T, V), generator=g, dtype=torch.int32)
        z[0] = 7
        z[1] = torch.arange(V, dtype=torch.int32)
        z[2] = -torch.arange(V, dtype=torch.int32)
        z[3] = -2 ** 31
        _compare(z, torch.randint(0, V, (T, 1), generator=g, dtype=torch.int32), 1 / 64, (5, 32))
