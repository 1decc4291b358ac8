"""The 8-bit and answering operators around the binary layers, each called as a
user's program calls it, over the range of its sizes.

A binarized network keeps some layers in more than one bit: its first and last
ones, and the projections that lose too much as signs.  A case names one
operator and its sizes.  ``listed()`` are the fixed points, ``draw(rng)`` gives
another point of the same ranges:

  norm      root-mean-square norm of the rows with the residual added on the
            way, and its output in 8-bit integers with a scale per row
  q8        matrix product of 8-bit integers with a scale per row (token) and
            per output (channel), and a bias
  logprobs  log probabilities of given answers (classes, tokens) from the last
            layer's logits, with the entropy and the largest alternatives

With ``own`` false, ``run`` computes them in plain 32-bit torch operations (64
bits for the 8-bit roundings, whose borders 32 bits would cross); with ``own``
true through the package's binding.  ``exact`` is the definition in 64 bits.

8-bit rows are laid out as the norm writes them and as a program lays out its
weights once: a multiple of 16 bytes apart.  Sizes: 1024 and 4096 inputs and
outputs are the FC layers of the tracked workloads (``perf/cases.py``), 1100
and 2050 those of their ragged tests; 65536 and 131072 answers are generic
vocabularies, 1000 a generic number of classes.
"""
import math

import torch

DEV = "cuda"
own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16, "int32": torch.int32}


# ------------------------------------------------------------------ cases ---
def listed():
    return [
        # One token between two layers: latency.
        dict(name="norm_1_4096", family="norm", M=1, D=4096, type="bf16", residual=True),
        # Ragged rows in 32 bits, a network's input without a residual.
        dict(name="norm_301_1100", family="norm", M=301, D=1100, type="fp32", residual=False),
        # A large prompt batch.
        dict(name="norm_8192_4096", family="norm", M=8192, D=4096, type="bf16", residual=True),
        # One token through one layer: the weights are all there is to read.
        dict(name="q8_1_4096_4096", family="q8", M=1, K=4096, N=4096, bias=False, out="bf16"),
        # The last layer of a decoding batch, one logit for each answer.
        dict(name="q8_16_4096_65536", family="q8", M=16, K=4096, N=65536, bias=False, out="fp32"),
        # A short prompt: too few tiles for the card if each keeps its whole sum.
        dict(name="q8_256_4096_4096", family="q8", M=256, K=4096, N=4096, bias=False, out="bf16"),
        # Ragged sizes in the middle of the range.
        dict(name="q8_777_1100_2050", family="q8", M=777, K=1100, N=2050, bias=True, out="fp32"),
        # A large prompt batch through a block's wide layer.
        dict(name="q8_8192_4096_16384", family="q8", M=8192, K=4096, N=16384, bias=False,
             out="bf16"),
        # The answer to one request: one row, a whole vocabulary.
        dict(name="logprobs_1_65536", family="logprobs", T=1, V=65536, type="bf16", n=1, top_k=20,
             masked=0.0),
        # A classifier's answers to a large batch, from a binary layer's sums.
        dict(name="logprobs_16384_1000", family="logprobs", T=16384, V=1000, type="int32", n=1,
             top_k=5, masked=0.0),
        # Ragged rows with answers out of reach and several candidates to score.
        dict(name="logprobs_301_50021", family="logprobs", T=301, V=50021, type="fp32", n=4,
             top_k=8, masked=0.1),
        # Scoring every token of a large prompt batch.
        dict(name="logprobs_4096_131072", family="logprobs", T=4096, V=131072, type="bf16", n=1,
             top_k=8, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    family = rng.choice(["norm", "q8", "logprobs"])
    if family == "norm":
        D = rng.choice([1024, 2048, 4096, 8192, _log(rng, 64, 16384)])
        return dict(family=family, M=min(_log(rng, 1, 65536), max(1, 4096 * 8192 // D)), D=D,
                    type=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    residual=rng.random() < 0.7)
    if family == "q8":
        K = rng.choice([1024, 2048, 4096, _log(rng, 64, 8192)])
        N = rng.choice([1024, 2048, 4096, 8192, _log(rng, 33, 65536)])
        N = min(N, 4096 * 65536 // K)
        M = min(_log(rng, 1, 8192), max(1, 8192 * 16384 * 4096 // (N * K)))
        return dict(family=family, M=M, K=K, N=N, bias=rng.random() < 0.3,
                    out=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    V = rng.choice([1000, 32768, 65536, _log(rng, 100, 131072)])
    kind = rng.choice(["bf16", "fp32", "fp16", "int32"])
    T = min(_log(rng, 1, 16384), (2048 if kind in ("fp32", "int32") else 4096) * 131072 // V)
    return dict(family=family, T=T, V=V, type=kind, n=rng.choice([1, 1, 4]),
                top_k=rng.choice([0, 1, 5, 8, 20]),
                masked=0.0 if kind == "int32" else rng.choice([0.0, 0.1, 0.9]))


# ----------------------------------------------------------------- inputs ---
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rows8(v):
    """8-bit values [M, K] in rows that are a multiple of 16 bytes apart."""
    M, K = v.shape
    rows = torch.zeros((M, (K + 15) // 16 * 16), dtype=torch.int8, device=v.device)
    rows[:, :K] = v
    return rows[:, :K]


def _quantized(v):
    """Rows of real values as 8-bit integers and their scales."""
    scale = v.abs().amax(1).clamp_min(1e-20) / 127
    return _rows8(torch.round(v / scale[:, None]).clamp(-127, 127).to(torch.int8)), scale


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=dict(case))
    family = case["family"]
    if family == "norm":
        # the stream of a deep network: a few channels much larger than the rest
        M, D, kind = case["M"], case["D"], TYPES[case["type"]]
        loud = 1 + 20.0 * (torch.rand(D, generator=g, device=DEV) < 0.01)
        s.update(x=_normal(g, M, D).to(kind), weight=(1 + 0.2 * _normal(g, D)).to(kind),
                 residual=(2 * loud * _normal(g, M, D)).to(kind) if case["residual"] else None)
    elif family == "q8":
        M, K, N = case["M"], case["K"], case["N"]
        x, x_scale = _quantized(_normal(g, M, K))
        w, w_scale = _quantized(_normal(g, N, K) / math.sqrt(K))
        s.update(x=x, x_scale=x_scale, w=w, w_scale=w_scale,
                 bias=0.1 * _normal(g, N) if case["bias"] else None)
    else:
        # rows of different sharpness over answers of different popularity;
        # `masked` of the answers are out of reach (-inf)
        T, V = case["T"], case["V"]
        sharp = torch.exp(0.7 * _normal(g, T, 1))
        z = _normal(g, T, V).mul_(sharp).add_(_normal(g, V))
        if case["type"] == "int32":
            z = 2 * torch.round(16 * z)  # sums of +-1 products
        if case["masked"]:
            z[torch.rand((T, V), generator=g, device=DEV) < case["masked"]] = -math.inf
        ids = torch.randint(0, V, (T, case["n"]), generator=g, device=DEV)
        s.update(logits=z.to(TYPES[case["type"]]), ids=ids.to(torch.int32),
                 scale=1.0 / 32 if case["type"] == "int32" else 1.0)
    return s


# -------------------------------------------------------------- plain forms ---
def _plain_norm(s):
    kind = s["x"].dtype
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(kind)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    p = h.double() * s["weight"].double()
    top = p.abs().amax(1)
    q = torch.round(p * 127 / top[:, None].clamp_min(1e-300))
    scale = (top * rstd / 127).float()
    return {"sum": h if s["residual"] is not None else None,
            "values": (q.float() * scale[:, None]).to(kind)}


def _plain_q8(s):
    y = (s["x"].float() @ s["w"].float().T) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(TYPES[s["case"]["out"]])


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() * s["scale"]
    top = z.amax(1, keepdim=True).clamp_min(-3e38)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    entropy = torch.log(total[:, 0]) - (e * (z - top).clamp_min(-1e4)).sum(1) / total[:, 0]
    out = {"logprobs": z.gather(1, s["ids"].long()) - lse, "entropy": entropy}
    if c["top_k"]:
        # equal logits go to the lowest index: value and index as one integer
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        bits = bits ^ ((bits >> 31) & 0x7fffffff)
        last = c["V"] - 1 - torch.arange(c["V"], device=z.device)
        best = (bits.long() * 2 ** 32 + last).topk(c["top_k"], dim=1).values
        ids = c["V"] - 1 - (best & 0xffffffff)
        best = z.gather(1, ids)
        out.update(top_ids=ids.masked_fill(torch.isneginf(best), -1).to(torch.int32),
                   top_logprobs=best - lse)
    return out


def run(s):
    c = s["case"]
    family = c["family"]
    if not own:
        return {"norm": _plain_norm, "q8": _plain_q8, "logprobs": _plain_logprobs}[family](s)
    from paper_1808_00209_amd import bnn
    if family == "norm":
        h, _, q, scale = bnn.bnn_rmsnorm(s["x"], s["weight"], s["residual"], eps=1e-6)
        # the 8-bit output as the values it stands for
        values = torch.empty(q.shape, dtype=s["x"].dtype, device=q.device)
        torch.mul(q, scale[:, None], out=values)
        return {"sum": h, "values": values}
    if family == "q8":
        return bnn.bnn_q8gemm(s["x"], s["w"], s["x_scale"], s["w_scale"], s["bias"],
                              dtype=TYPES[c["out"]])
    given, entropy, top_ids, top = bnn.bnn_logprobs(s["logits"], s["ids"], top_k=c["top_k"],
                                                    logit_scale=s["scale"])
    out = {"logprobs": given, "entropy": entropy}
    if c["top_k"]:
        out.update(top_ids=top_ids, top_logprobs=top)
    return out


# ------------------------------------------------------------------- work ---
def work(case):
    family = case["family"]
    if family == "norm":
        M, D = case["M"], case["D"]
        size = 4 if case["type"] == "fp32" else 2
        return {"bytes": M * D * (size * (3 if case["residual"] else 1) + 1) + 4 * M + D * size,
                "flops": 6 * M * D}
    if family == "q8":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": (M + N) * (K + 4) + M * N * (4 if case["out"] == "fp32" else 2)
                + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    T, V = case["T"], case["V"]
    size = 2 if case["type"] in ("bf16", "fp16") else 4
    return {"bytes": T * V * size + T * (8 * case["n"] + 4 + 8 * case["top_k"]),
            "flops": 5 * T * V}


# ------------------------------------------------- the definition, 64 bits ---
def exact(case, seed):
    s = prepare(case, seed)
    family = case["family"]
    if family == "norm":
        x = s["x"].double()
        if s["residual"] is not None:  # the sum is kept in the stream's type
            x = (x + s["residual"].double()).to(s["x"].dtype).double()
        y = x / torch.sqrt((x * x).sum(1, keepdim=True) / case["D"] + 1e-6) * s["weight"].double()
        step = torch.max(torch.abs(y), dim=1, keepdim=True).values / 127
        n = torch.abs(x * s["weight"].double())
        n = n / torch.max(n, dim=1, keepdim=True).values * 127
        whole = torch.floor(n)
        up = (n - whole > 0.5) | ((n - whole == 0.5) & (whole % 2 == 1))
        values = torch.sign(y) * (whole + up) * step
        return {"sum": x if s["residual"] is not None else None, "values": values}
    if family == "q8":
        a = s["x"].double() * s["x_scale"].double()[:, None]
        y = torch.cat([a @ (part.double() * scale.double()[:, None]).T for part, scale in
                       zip(s["w"].split(4096), s["w_scale"].split(4096))], dim=1)
        return y if s["bias"] is None else y + s["bias"].double()
    parts = []
    for z, ids in zip(s["logits"].split(256), s["ids"].split(256)):
        z = z.double() * s["scale"]
        lp = torch.log_softmax(z, dim=1)
        p = torch.exp(lp)
        part = [lp.gather(1, ids.long()), -torch.where(p > 0, p * lp, 0.0).sum(1)]
        if case["top_k"]:
            best, at = torch.sort(lp, dim=1, descending=True, stable=True)
            best, at = best[:, :case["top_k"]], at[:, :case["top_k"]]
            part += [torch.where(torch.isneginf(best), -1, at).to(torch.int32), best]
        parts.append(part)
    return dict(zip(("logprobs", "entropy", "top_ids", "top_logprobs"),
                    (torch.cat(v) for v in zip(*parts))))
