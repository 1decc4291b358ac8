"""The mixture-of-experts calls in 64 bits on the CPU, written from their
definitions in include/bnn.h: what the kernels are compared with."""
import numpy as np


def pm1(words, D):
    """Packed words [..., ceil(D/32)] (any 32-bit integers) -> +-1 [..., D]."""
    w = np.asarray(words).astype(np.int64) & 0xFFFFFFFF
    i = np.arange(D)
    return ((w[..., i // 32] >> (31 - i % 32)) & 1) * 2 - 1


def pack(bits):
    """Truth values [..., D] -> int32 words, tail bits 0."""
    b = np.asarray(bits, dtype=np.uint8)
    pad = -b.shape[-1] % 32
    b = np.concatenate([b, np.zeros((*b.shape[:-1], pad), np.uint8)], axis=-1)
    by = np.packbits(b, axis=-1).reshape(*b.shape[:-1], -1, 4).astype(np.uint32)
    w = by[..., 0] << 24 | by[..., 1] << 16 | by[..., 2] << 8 | by[..., 3]
    return w.view(np.int32)


def route(logits, top_k, bias=None, score="softmax", groups=1, top_groups=None, group_top=1,
          renorm=True, scale=1.0, logit_scale=1.0):
    """ids, weights, and how near the closest unequal keys that the choice
    hangs on come to each other."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    top_groups = groups if top_groups is None else top_groups
    ids, weights = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k))
    near = np.inf
    big = float(np.finfo(np.float32).max)

    def ranked(v, n):
        nonlocal near
        at = sorted((i for i in range(len(v)) if v[i] > -np.inf), key=lambda i: (-v[i], i))
        gaps = [v[a] - v[b] for a, b in zip(at[:n], at[1:n + 1]) if v[a] != v[b]]
        near = min([near] + gaps)
        return at[:n]

    for t in range(T):
        z = np.clip(x[t] * logit_scale, -big, big)
        out = ~(x[t] > -np.inf)
        z[out] = -np.inf
        p = np.zeros(E)
        if not out.all():
            if score == "softmax":
                e = np.where(out, 0.0, np.exp(z - z[~out].max()))
                p = e / e.sum()
            else:
                with np.errstate(over="ignore"):
                    p = 1 / (1 + np.exp(-z))
        key = p + (0.0 if bias is None else np.asarray(bias, np.float64))
        key = np.where(out | ~(key > -np.inf), -np.inf, key)
        if groups > 1:
            per = E // groups
            gs = np.full(groups, -np.inf)
            for g in range(groups):
                best = sorted(key[g * per:(g + 1) * per], reverse=True)[:group_top]
                best = [v for v in best if v > -np.inf]
                if best:
                    gs[g] = sum(best)
            keep = ranked(gs, top_groups)
            mask = np.repeat(np.isin(np.arange(groups), keep), per)
            key = np.where(mask, key, -np.inf)
        at = ranked(key, top_k)
        w = p[at]
        if renorm and w.sum() > 0:
            w = w / w.sum()
        ids[t, :len(at)], weights[t, :len(at)] = at, scale * w
    return ids, weights, near


def group_rows(ids, G):
    ids = np.asarray(ids).reshape(-1).astype(np.int64)
    g = np.where((ids >= 0) & (ids < G), ids, G)
    offsets = np.searchsorted(np.sort(g), np.arange(G + 1), side="left")
    return offsets.astype(np.int32), np.argsort(g, kind="stable").astype(np.int32)


def expert_sums(x, w, ids, K):
    """int sums [M, N] of pairs m: row m // (M / rows of x) with expert ids[m]."""
    ids = np.asarray(ids).reshape(-1)
    X = pm1(x, K)
    share = len(ids) // len(X)
    S = np.zeros((len(ids), w.shape[1]), np.int64)
    for e in range(w.shape[0]):
        at = np.nonzero(ids == e)[0]
        if len(at):
            a, b = X[at // share].astype(np.float64), pm1(w[e], K).astype(np.float64)
            S[at] = (a @ b.T).astype(np.int64)
    return S


def experts_fc(x, w, ids, K, thr, flip=None):
    ids = np.asarray(ids).reshape(-1)
    S, N, E = expert_sums(x, w, ids, K), w.shape[1], w.shape[0]
    safe = np.clip(ids, 0, E - 1)
    bits = S >= np.asarray(thr).astype(np.int64)[safe]
    if flip is not None:
        bits ^= pm1(flip, N)[safe] > 0
    return pack(bits & ((ids >= 0) & (ids < E))[:, None])


def experts_sum(x, w, ids, weights, K, alpha=None):
    """y [T, N] and the sum of the magnitudes that it adds up."""
    T, k = ids.shape
    E, N = w.shape[:2]
    S = expert_sums(x, w, ids, K).reshape(T, k, N).astype(np.float64)
    safe = np.clip(ids, 0, E - 1)
    al = np.ones((E, N)) if alpha is None else np.asarray(alpha, np.float64)
    on = ((ids >= 0) & (ids < E))[..., None]
    part = np.where(on, np.where(on, weights[..., None], 0.0).astype(np.float64) * al[safe] * S, 0.0)
    return part.sum(1), np.abs(part).sum(1)


def lora(x, w, ids, a, b, scale=None, alpha=None, offset=None):
    """y [M, N], |alpha S|, and the magnitudes that the adapter's term adds up."""
    x, a, b = (np.asarray(v, np.float64) for v in (x, a, b))
    M, K = x.shape
    N = w.shape[0]
    off = 0.0 if offset is None else np.asarray(offset, np.float64)
    base = np.where(x + off > 0, 1.0, -1.0) @ pm1(w, K).astype(np.float64).T
    if alpha is not None:
        base = base * np.asarray(alpha, np.float64)
    add, mag = np.zeros((M, N)), np.zeros((M, N))
    for l in range(a.shape[0]):
        at = np.nonzero(np.asarray(ids) == l)[0]
        if len(at):
            s = 1.0 if scale is None else float(scale[l])
            add[at] = s * (x[at] @ a[l].T) @ b[l].T
            mag[at] = abs(s) * (np.abs(x[at]) @ np.abs(a[l]).T) @ np.abs(b[l]).T
    return base + add, np.abs(base), mag
