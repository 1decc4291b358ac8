"""Routing and the order of rows by group, against their definitions in 64
bits (experts_ref).

Tolerances.  A weight passes through z = logit * scale (exact here: powers of
two), expf of an argument of at most 50 (its rounding moves the result by at
most 50 * 2^-24 relative, expf itself by 2 units), a sum of at most 1024
positive terms in at most 16 + 6 additions one after another, two divisions
and one product: under 90 * 2^-24 < 1e-5 relative, and the sum of the chosen
ones as much again: 2e-5.  Below 2^-126 only the absolute 1e-30 is asked."""
import numpy as np
import pytest
import torch

import experts_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

NEAR = 1e-5  # keys nearer than this to each other would leave the choice open
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16,
         "int32": torch.int32}


def _check(logits, top_k, bias=None, near=NEAR, **kw):
    """logits: a host tensor."""
    dev = logits.cuda()
    b = None if bias is None else torch.from_numpy(np.asarray(bias, np.float32)).cuda()
    ids, w = bnn.bnn_route(dev, top_k, b, **kw)
    torch.cuda.synchronize()
    r = dict(kw)
    r["renorm"] = r.pop("renormalize", True)
    rid, rw, gap = ref.route(logits.double().numpy(), top_k, bias, **r)
    assert gap > near, "the case leaves the choice open"
    assert np.array_equal(ids.cpu().numpy(), rid)
    np.testing.assert_allclose(w.cpu().numpy(), rw, rtol=2e-5, atol=1e-30)


CASES = [
    # T, E, top_k, groups, top_groups, group_top, score, bias, type, renorm
    (1, 1, 1, 1, 1, 1, "softmax", 0, "fp32", 1), (3, 4, 2, 1, 1, 1, "sigmoid", 1, "bf16", 1),
    (5, 8, 8, 1, 1, 1, "softmax", 1, "fp16", 0), (1, 64, 8, 1, 1, 1, "softmax", 0, "bf16", 1),
    (7, 60, 6, 1, 1, 1, "softmax", 0, "int32", 0), (67, 64, 8, 8, 3, 2, "sigmoid", 1, "fp32", 1),
    (17, 65, 1, 5, 2, 1, "softmax", 0, "fp32", 0), (33, 128, 4, 4, 1, 2, "softmax", 1, "bf16", 1),
    (50, 256, 8, 8, 4, 2, "sigmoid", 1, "fp32", 1), (9, 160, 6, 8, 3, 1, "softmax", 0, "fp32", 1),
    (4, 257, 16, 1, 1, 1, "softmax", 0, "fp16", 1), (6, 384, 8, 64, 9, 2, "sigmoid", 1, "fp32", 0),
    (2, 1000, 16, 8, 3, 2, "softmax", 1, "fp32", 1), (3, 1024, 10, 1, 1, 1, "sigmoid", 0, "fp32", 1),
    (31, 12, 3, 12, 4, 2, "softmax", 0, "bf16", 1), (300, 16, 2, 1, 1, 1, "softmax", 0, "int32", 1),
    (129, 33, 5, 3, 2, 2, "sigmoid", 1, "fp16", 1), (70, 512, 7, 16, 16, 1, "softmax", 0, "bf16", 1),
]


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%d-%d-%d-%s-%s" % (c[0], c[1], c[2], c[6], c[8]))
def test_route(case, masked):
    T, E, k, groups, top_groups, group_top, score, bias, kind, renorm = case
    g = np.random.default_rng(1000 * E + T)
    # Scores on a grid of 1/8 and biases on one of 1/64 that no difference of
    # two scores comes near: equal keys are equal in 32 bits, others far apart.
    x = torch.from_numpy(g.integers(-24, 25, size=(T, E)) / 8.0)
    b = g.integers(-8, 9, size=E) / 64.0 if bias else None
    if kind == "int32":
        x, kw = (x * 8).to(torch.int32), dict(logit_scale=0.125)
    else:
        x, kw = x.to(TYPES[kind]), {}
        x[torch.from_numpy(g.random((T, E)) < masked)] = -float("inf")
        x[torch.from_numpy(g.random(T) < masked / 4)] = -float("inf")
    _check(x, k, b, near=1e-6, score=score, groups=groups, top_groups=top_groups,
           group_top=group_top, renormalize=bool(renorm), scale=2.5, **kw)


def test_ties_go_to_the_lowest_index():
    for E in (5, 64, 100, 256, 300, 1024):
        x = torch.zeros(3, E)
        x[1, E // 2:] = 1.0
        x[2, E - 1] = 1.0
        _check(x, min(E, 9))
        _check(x, min(E, 9), score="sigmoid")


@pytest.mark.parametrize("E", [16, 60, 128, 250, 256, 640, 1024])
def test_few_distinct_keys(E):
    # Runs of equal keys that begin and end anywhere, longer and shorter than
    # what is held ready of one stretch of experts, closed ones between them.
    g = np.random.default_rng(E)
    x = g.integers(0, 3, size=(40, E)).astype(np.float32)
    for t in range(0, 40, 2):
        x[t] = 0.0
        at = int(g.integers(0, E))
        x[t, at:at + int(g.integers(1, 20))] = 1.0
    x[g.random((40, E)) < 0.2] = -float("inf")
    x = torch.from_numpy(x)
    for k in (1, 5, min(E, 16)):
        _check(x, k)
        _check(x, k, score="sigmoid")
        _check(x, k, score="sigmoid", groups=2, top_groups=1, group_top=2)


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
def test_the_lowest_value_is_no_mask_and_minus_infinity_is(kind):
    t = TYPES[kind]
    low, inf = torch.finfo(t).min, float("inf")
    x = torch.tensor([[low, low, low, low], [-inf, low, -inf, low], [-inf] * 4,
                      [-inf, -inf, 3.0, -inf], [low, 0.5, -inf, low], [float("nan")] * 4,
                      [float("nan"), 1.0, -inf, 2.0]], dtype=t)
    for score in ("softmax", "sigmoid"):
        for k in (1, 3, 4):
            _check(x, k, score=score)
            _check(x, k, score=score, groups=2, top_groups=1, group_top=2)
    ids, w = bnn.bnn_route(x.cuda(), 3)
    assert ids[2].tolist() == [-1, -1, -1] and w[2].tolist() == [0.0, 0.0, 0.0]
    assert ids[3].tolist() == [2, -1, -1] and w[3].tolist() == [1.0, 0.0, 0.0]
    assert ids[0].tolist() == [0, 1, 2]


def test_infinite_logits_scores_that_vanish_and_scales_that_overflow():
    inf = float("inf")
    x = torch.tensor([[inf, 0.0, inf, 1.0], [0.0, 0.0, 0.0, inf], [-200.0, -300.0, -200.0, -150.0],
                      [3e38, -3e38, 1e38, 3e38]])
    ids, w = bnn.bnn_route(x.cuda(), 2)
    assert ids.tolist() == [[0, 2], [3, 0], [3, 0], [0, 3]]
    assert torch.allclose(w[0].cpu(), torch.tensor([0.5, 0.5])) and w[1].tolist() == [1.0, 0.0]
    ids, w = bnn.bnn_route(x.cuda(), 2, score="sigmoid")
    assert ids[2].tolist() == [3, 0] or ids[2].tolist() == [0, 1]  # (all vanish in 32 bits)
    assert torch.isfinite(w).all() and (w[2] >= 0).all()
    ids, w = bnn.bnn_route(x.cuda(), 4, logit_scale=1e20)
    assert torch.isfinite(w).all() and sorted(ids[3].tolist()) == [0, 1, 2, 3]


def test_a_bias_chooses_but_does_not_weigh_and_one_of_minus_infinity_closes():
    x = torch.zeros(2, 6)
    b = np.array([0, 0, 5, -np.inf, np.nan, 1], np.float32)
    ids, w = bnn.bnn_route(x.cuda(), 4, torch.from_numpy(b).cuda(), renormalize=False)
    assert ids.tolist() == [[2, 5, 0, 1]] * 2
    assert torch.allclose(w.cpu(), torch.full((2, 4), 1 / 6))
    ids, w = bnn.bnn_route(x.cuda(), 5, torch.from_numpy(b).cuda())
    assert ids[0].tolist() == [2, 5, 0, 1, -1] and w[0, 4] == 0


def test_strided_rows_and_no_rows():
    g = np.random.default_rng(5)
    x = torch.from_numpy(g.integers(-24, 25, size=(9, 70)) / 8.0).float()
    wide = torch.full((9, 101), 99.0)
    wide[:, :70] = x
    ids, w = bnn.bnn_route(wide.cuda()[:, :70], 5)
    ids2, w2 = bnn.bnn_route(x.cuda(), 5)
    assert torch.equal(ids, ids2) and torch.equal(w, w2)
    odd = wide.to(torch.bfloat16).cuda()[:, 1:70]  # rows of odd distance, 2-byte aligned
    ids, w = bnn.bnn_route(odd, 5)
    ids2, w2 = bnn.bnn_route(odd.contiguous(), 5)
    assert torch.equal(ids, ids2) and torch.equal(w, w2)
    ids, w = bnn.bnn_route(torch.empty(0, 8, device="cuda"), 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)


GROUP_CASES = [(0, 1), (1, 1), (1, 1024), (63, 5), (64, 64), (65, 2), (1000, 256), (1023, 7),
               (1024, 7), (1025, 7), (5000, 1000), (8192, 64), (70001, 33), (262144, 8),
               (131072, 256), (300000, 300), (16384, 100), (16385, 1023), (20000, 1024), (3000001, 77)]


@pytest.mark.parametrize("M, G", GROUP_CASES, ids=str)
@pytest.mark.parametrize("how", ["even", "outside", "skewed", "one"])
def test_group_rows(M, G, how):
    g = np.random.default_rng(M + G)
    ids = g.integers(0, G, size=M)
    if how == "outside":
        ids = np.where(g.random(M) < 0.3, g.choice([-1, G, 2 ** 31 - 1, -2 ** 31], size=M), ids)
    elif how == "skewed":
        ids = (G * g.random(M) ** 6).astype(np.int64)
    elif how == "one":
        ids[:] = G - 1
    ids = ids.astype(np.int32)
    offsets, order = bnn.bnn_group_rows(torch.from_numpy(ids).cuda(), G)
    torch.cuda.synchronize()
    want = ref.group_rows(ids, G)
    assert np.array_equal(offsets.cpu().numpy(), want[0])
    assert np.array_equal(order.cpu().numpy(), want[1])
