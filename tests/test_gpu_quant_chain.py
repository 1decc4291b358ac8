"""The norm, the 8-bit product and the log probabilities one after another, as a
program runs them behind its last binary layers; captured and replayed, on other
streams, with shared workspaces."""
import math

import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu


def _made(T, D, H, V, kind, seed):
    g = torch.Generator().manual_seed(seed)
    rows = lambda n, k, s=1.0: (s * torch.randn(n, k, generator=g)).to(kind)  # noqa: E731

    def weights(n, k):  # laid out once: 8 bits, rows a multiple of 16 bytes apart, a scale each
        w = torch.randn(n, k, generator=g) / math.sqrt(k)
        scale = w.abs().amax(1) / 127
        q = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.int8)
        q[:, :k] = torch.round(w / scale[:, None]).to(torch.int8)
        return q[:, :k], scale

    w1, s1 = weights(H, D)
    w2, s2 = weights(V, H)
    return dict(x=rows(T, D), r=rows(T, D, 2.0), n1=rows(1, D)[0], n2=rows(1, H)[0], w1=w1, s1=s1, w2=w2, s2=s2,
                ids=torch.randint(0, V, (T, 2), generator=g, dtype=torch.int32))


def _device(m):
    out = {k: v.cuda() for k, v in m.items() if not k.startswith("w")}
    for k in ("w1", "w2"):
        store = torch.zeros(m[k].shape[0], m[k].stride(0), dtype=torch.int8, device="cuda")
        out[k] = store[:, :m[k].shape[1]]
        out[k].copy_(m[k])
    return out


def _run(d, workspace=None, stream=None):
    kind = d["x"].dtype
    h, _, q, s = bnn.bnn_rmsnorm(d["x"], d["n1"], d["r"], eps=1e-5, stream=stream)
    y = bnn.bnn_q8gemm(q, d["w1"], s, d["s1"], dtype=kind, stream=stream)
    _, _, q2, s2 = bnn.bnn_rmsnorm(y, d["n2"], eps=1e-5, stream=stream)
    z = bnn.bnn_q8gemm(q2, d["w2"], s2, d["s2"], dtype=torch.float32, stream=stream)
    return (h, y, z) + bnn.bnn_logprobs(z, d["ids"], 6, workspace=workspace, stream=stream)


@pytest.mark.parametrize("T, D, H, V, kind", [
    (1, 1024, 1000, 10007, torch.bfloat16), (5, 100, 333, 70, torch.float16), (70, 512, 1024, 1000, torch.bfloat16),
    (300, 1100, 700, 5000, torch.float32), (40, 33, 17, 9000, torch.bfloat16)])
def test_chain(T, D, H, V, kind):
    m = _made(T, D, H, V, kind, D + T)
    h, y, z, given, entropy, top_ids, top = (t.cpu() for t in _run(_device(m)))
    # In 64 bits.  y is kept in `kind`: it is taken as the kernels gave it after
    # a comparison (one rounding more than the definition, and the scale's).
    hr, _, q, s = ref.rmsnorm(m["x"], m["n1"], m["r"], 1e-5)
    yr = (q.double() @ m["w1"].double().T) * s[:, None] * m["s1"].double()
    assert torch.equal(h, hr)
    torch.testing.assert_close(y.double(), yr, rtol=50 * 2.0 ** -24 + torch.finfo(kind).eps / 2, atol=1e-7)
    _, _, q, s = ref.rmsnorm(y, m["n2"], None, 1e-5)
    zr = (q.double() @ m["w2"].double().T) * s[:, None] * m["s2"].double()
    torch.testing.assert_close(z.double(), zr, rtol=50 * 2.0 ** -24, atol=1e-30)
    g, e, _, _ = ref.logprobs(zr, m["ids"], 0)
    # an error of 50 * 2^-24 of the largest logit in every logit moves ln p and
    # the entropy (whose gradient is at most 1 + ln V) by as much, beside their
    # own roundings
    off = 50 * 2.0 ** -24 * zr.abs().max().item()
    own = 2.0 ** -24 * (3 * (g.abs().max().item() + 1) + V / 512 + 200)
    assert (given.double() - g).abs().max() <= 2 * off + own
    assert (entropy.double() - e).abs().max() <= (2 * off + own) * (3 + math.log(V))
    _, _, ti, tl = ref.logprobs(z, None, 6)
    assert torch.equal(top_ids, ti)
    assert (top.double() - tl).abs().max() <= own


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T, D, H, V", [(1, 1024, 1024, 20000), (200, 512, 2048, 4100), (3, 4096, 1000, 70000)])
def test_captured(T, D, H, V):
    """Replayed on new inputs, with eager work between, bit by bit as eagerly."""
    d = _device(_made(T, D, H, V, torch.bfloat16, 3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(d)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _run(d)
    for seed in range(4):
        new = _device(_made(T, D, H, V, torch.bfloat16, 50 + seed))
        for k in d:
            d[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        assert _equal(kept, _run(new)), seed
        junk = torch.full((1 << 22,), float(seed), device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        assert _equal(kept, out) and junk.sum().item() == seed * float(1 << 22)


def test_two_graphs_share_a_workspace():
    """One after another on a stream: each writes the workspace before it reads."""
    T, V = 3, 50000
    size = bnn.bnn_logprobs_workspace_size(bnn.LogprobsDesc(64, V, 2, 6, 0, 1.0))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    ds = [_device(_made(t, 256, 500, V, torch.bfloat16, 7 + t)) for t in (T, 20)]
    want = [[t.clone() for t in _run(d)] for d in ds]
    graphs, outs = [], []
    for d in ds:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(_run(d, workspace=ws))
        graphs.append(graph)
    for _ in range(3):
        ws.fill_(0xA5)
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        assert all(_equal(o, w) for o, w in zip(outs, want))


def test_streams():
    """On a stream of the caller's, and on two at once."""
    ds = [_device(_made(t, 700, 900, 30000, torch.float16, 11 + t)) for t in (4, 90)]
    want = [[t.clone() for t in _run(d)] for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ds]
    for _ in range(5):
        outs = [_run(d, stream=s) for d, s in zip(ds, streams)]
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(_equal(o, w) for o, w in zip(outs, want))
        with torch.cuda.stream(streams[0]):
            inside = _run(ds[1])
        torch.cuda.current_stream().wait_stream(streams[0])
        assert _equal(inside, want[1])


def test_binary_sums_as_logits():
    """A binary layer's int32 sums, as the classifier's last layer gives them."""
    g = torch.Generator().manual_seed(2)
    a = torch.randint(-2 ** 31, 2 ** 31, (50, 32), generator=g, dtype=torch.int64).to(torch.int32)
    b = torch.randint(-2 ** 31, 2 ** 31, (1000, 32), generator=g, dtype=torch.int64).to(torch.int32)
    sums, _ = bnn.bnn_bgemm(a.cuda(), b.cuda(), 1024, want_bits=False)
    ids = torch.randint(0, 1000, (50,), generator=g, dtype=torch.int32)
    lp, entropy, top_ids, top = (t.cpu() for t in bnn.bnn_logprobs(sums, ids.cuda(), 5, logit_scale=1 / 32))
    r = ref.logprobs(sums.cpu(), ids, 5, 1 / 32)
    assert torch.equal(top_ids, r[2])
    tol = 2.0 ** -24 * (3 * 20 + 202)
    for x, y, f in ((lp, r[0], 1), (entropy, r[1], 3 + math.log(1000)), (top, r[3], 1)):
        assert (x.double() - y).abs().max() <= tol * f
