"""The mixture-of-experts calls one after another (examples/expert_block.py):
every step against its 64-bit definition on what the step before gave, as one
HIP graph replayed on new inputs, and the vector-ALU forms of the calls."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import experts_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "expert_block", os.path.join(ROOT, "examples", "expert_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _block():
    return _example().ExpertBlock(width=256, hidden=512, experts=16, top_k=4, groups=4,
                                  top_groups=2, adapters=5, rank=8, seed=3)


def _inputs(T, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((T, 256), generator=g, device="cuda").to(torch.bfloat16)
    return h, torch.randint(-1, 5, (T,), generator=g, device="cuda").to(torch.int32)


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


@pytest.mark.parametrize("T", [1, 7, 64, 1500])
def test_every_step_against_its_definition(T):
    block = _block()
    h, adapter = _inputs(T, T)
    d = {}
    out = block(h, adapter, d)
    torch.cuda.synchronize()
    on = _np(h.float()) + _np(block.offset) > 0
    assert np.array_equal(_np(d["bits"]), ref.pack(on))
    x, w = ref.pm1(_np(d["bits"]), 256), ref.pm1(_np(block.router), 256)
    assert np.array_equal(_np(d["scores"]), x @ w.T)
    ids, weights, near = ref.route(_np(d["scores"]), 4, _np(block.balance), score="sigmoid",
                                   groups=4, top_groups=2, group_top=2, logit_scale=1 / 32)
    same = (_np(d["ids"]) == ids).all(1)
    assert same.all() or near < 1e-5  # (the rows whose keys are that near may differ)
    assert same.mean() > 0.99
    np.testing.assert_allclose(_np(d["weights"])[same], weights[same], rtol=2e-5)
    got = _np(d["ids"])
    assert np.array_equal(_np(d["inner"]), ref.experts_fc(
        _np(d["bits"]), _np(block.w0), got, 256, _np(block.thr0), _np(block.flip0)))
    y, mag = ref.experts_sum(_np(d["inner"]), _np(block.w1), got, _np(d["weights"]), 512,
                             _np(block.alpha1))
    bound = 7 * 2.0 ** -24 * mag
    assert (np.abs(_np(d["routed"]) - y) <= bound + 2.0 ** -8 * (np.abs(y) + bound)).all()
    y, base, mag = ref.lora(_np(h), _np(block.shared), _np(adapter), _np(block.a), _np(block.b),
                            _np(block.adapter_scale), _np(block.alpha), _np(block.offset))
    bound = 2 * 2.0 ** -24 * base + (256 + 16) * 2.0 ** -24 * mag
    assert (np.abs(_np(d["shared"]) - y) <= bound + 2.0 ** -8 * (np.abs(y) + bound)).all()
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("T", [2, 300])
def test_as_a_graph(T):
    """Captured once, replayed on new inputs with eager work in between: every
    replay gives the eager call's bits."""
    block = _block()
    h, adapter = _inputs(T, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block(h, adapter)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(h, adapter)
    for seed in (2, 3, 4, 5):
        h2, a2 = _inputs(T, seed)
        h.copy_(h2)
        adapter.copy_(a2)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, block(h2, a2))
        torch.cuda.synchronize()


def test_the_vector_kernels_give_the_same():
    """algo = VALU: bits are the same, sums within the roundings of both."""
    block = _block()
    for T in (3, 200):
        h, adapter = _inputs(T, 40 + T)
        a, b = {}, {}
        block(h, adapter, a)
        with bnn.options(algo=bnn.ALGO_VALU):
            block(h, adapter, b)
        torch.cuda.synchronize()
        for k in ("bits", "scores", "ids", "weights", "inner"):
            assert torch.equal(a[k], b[k]), k
        for k in ("routed", "shared"):
            x, y = a[k].double(), b[k].double()
            assert ((x - y).abs() <= 2.0 ** -7 * y.abs() + 1e-6).all(), k


def test_rows_of_over_four_gigabytes():
    """Packed rows beyond 4 GiB: the first, the last and some between."""
    K, T, N = 65535, 524353, 2
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.empty((T, 2048), dtype=torch.int32, device="cuda").random_(generator=g)
    assert x.numel() * 4 > 1 << 32
    w = torch.empty((3, N, 2048), dtype=torch.int32, device="cuda").random_(generator=g)
    ids = torch.randint(0, 3, (T, 1), generator=g, device="cuda").to(torch.int32)
    thr = torch.zeros((3, N), dtype=torch.int32, device="cuda")
    offsets, order = bnn.bnn_group_rows(ids, 3)
    bits = bnn.bnn_experts_fc(x, K, w, offsets, order, thr)
    y = bnn.bnn_experts_sum(x, K, w, ids, torch.ones((T, 1), device="cuda"), offsets, order)
    at = [0, 1, 300001, T - 2, T - 1]
    S = ref.expert_sums(x[at].cpu().numpy(), w.cpu().numpy(), ids[at].cpu().numpy(), K)
    assert np.array_equal(y[at].cpu().numpy(), S)
    assert np.array_equal(bits[at].cpu().numpy(), ref.pack(S >= 0))
