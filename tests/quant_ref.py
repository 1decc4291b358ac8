"""The 8-bit layers and the answers' log probabilities in 64 bits on the CPU,
written from their definitions in include/bnn.h: what the kernels are compared
with."""
import numpy as np
import torch


def rmsnorm(x, weight=None, residual=None, eps=1e-6):
    """Host tensors -> h (of x's type), y and scale (float64), q (int8)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    v = h.double()
    w = torch.ones(x.shape[1], dtype=torch.float64) if weight is None else weight.double()
    eps = float(np.float32(eps))
    root = torch.sqrt((v * v).sum(1) / x.shape[1] + eps)
    r = torch.where(root > 0, 1 / root, torch.zeros_like(root))
    p = v * w
    top = p.abs().amax(1)
    bad = ~torch.isfinite(v).all(1)
    q = torch.round(127 * p / torch.where(top > 0, top, torch.ones_like(top))[:, None])
    q = torch.where(bad[:, None], torch.zeros_like(q), q)
    nan = float("nan")
    y = torch.where(bad[:, None], torch.full_like(p, nan), p * r[:, None])
    scale = torch.where(bad, torch.full_like(r, nan), top * r / 127)
    return h, y, q.to(torch.int8), scale


def q8gemm(x, w, x_scale=None, w_scale=None, bias=None, dtype=torch.float32):
    """Host tensors; the sums exact, the rest in the stated fp32 steps."""
    s = (x.double() @ w.double().T).float()  # |S| < 2^31: exact in 64 bits
    y = s * (torch.ones(x.shape[0]) if x_scale is None else x_scale)[:, None]
    y = y * (torch.ones(w.shape[0]) if w_scale is None else w_scale)
    return (y if bias is None else y + bias).to(dtype)


def logprobs(logits, ids=None, top_k=0, logit_scale=1.0):
    """Host tensors -> ln p of ids, entropy, top ids, their ln p (float64)."""
    raw = logits.double()
    z = raw * float(np.float32(logit_scale))
    T, V = z.shape
    bad = torch.isnan(z).any(1) | (z == float("inf")).any(1)
    none = (z == -float("inf")).all(1)
    lp = torch.log_softmax(z, dim=1)
    lp[none] = -float("inf")
    lp[bad] = float("nan")
    p = torch.exp(lp)
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    entropy[bad] = float("nan")
    given = None
    if ids is not None:
        at = ids.long().reshape(T, -1)
        there = (at >= 0) & (at < V)
        given = lp.gather(1, at.clamp(0, V - 1))
        given[~there] = -float("inf")
        given = given.reshape(ids.shape)
    top_ids = torch.full((T, top_k), -1, dtype=torch.int32)
    top = torch.full((T, top_k), -float("inf"), dtype=torch.float64)
    for t in range(T if top_k else 0):
        if bad[t]:
            top[t] = float("nan")
            continue
        order = torch.sort(raw[t], descending=True, stable=True).indices[:top_k]
        order = order[raw[t][order] > -float("inf")]
        top_ids[t, :len(order)] = order.to(torch.int32)
        top[t, :len(order)] = lp[t][order]
    return given, entropy, top_ids, top
