"""A residual block whose layers are binary, with experts and adapters: the
calls of a mixture of binary experts one after another, as a server runs them.

    python examples/expert_block.py [rows]

``ExpertBlock`` computes, for rows h [T, D] of requests that each may have an
adapter,

    s  = shared binary layer of h with the request's low-rank adapter
    e  = the row's top_k experts: binary layer, threshold, binary layer,
         weighted by the router
    out = h + s + e

where the router's scores are themselves sums of a binary layer.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1808_00209_amd import bnn  # noqa: E402


def random_words(g, *shape):
    """Packed +-1 weights (int32 storage), Bernoulli(0.5)."""
    return torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda",
                         dtype=torch.int64).to(torch.int32)


class ExpertBlock:
    """Weights of one block (random ones here), on the GPU."""

    def __init__(self, width=1024, hidden=4096, experts=64, top_k=8, groups=8, top_groups=4,
                 adapters=16, rank=16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.hidden, self.experts, self.top_k = width, hidden, experts, top_k
        self.groups, self.top_groups = groups, top_groups
        scale = lambda *s: (0.5 + torch.rand(s, generator=g, device="cuda")) / math.sqrt(s[-1])  # noqa: E731
        kw, hw = bnn.words(width), bnn.words(hidden)
        self.router = random_words(g, experts, kw)
        self.balance = 0.01 * torch.randn(experts, generator=g, device="cuda")
        r = 2 * math.isqrt(width)
        self.w0 = random_words(g, experts, hidden, kw)
        self.thr0 = torch.randint(-r, r + 1, (experts, hidden), generator=g,
                                  device="cuda").to(torch.int32)
        self.flip0 = random_words(g, experts, hw)
        self.w1, self.alpha1 = random_words(g, experts, width, hw), scale(experts, width)
        self.shared, self.alpha = random_words(g, width, kw), scale(width)
        self.offset = 0.1 * torch.randn(width, generator=g, device="cuda")
        self.a = torch.randn((adapters, rank, width), generator=g, device="cuda") / math.sqrt(width)
        self.b = torch.randn((adapters, width, rank), generator=g, device="cuda") / 8
        self.a, self.b = self.a.to(torch.bfloat16), self.b.to(torch.bfloat16)
        self.adapter_scale = torch.full((adapters,), 1 / math.sqrt(rank), device="cuda")

    def __call__(self, h, adapter, details=None):
        """h [T, width] bfloat16, adapter [T] int32 (-1: none) -> [T, width]
        bfloat16.  details: a dict that receives the steps' results."""
        bits = bnn.bnn_pack_bits(h.float(), self.offset)
        scores, _ = bnn.bnn_bgemm(bits, self.router, self.width, want_bits=False)
        ids, weights = bnn.bnn_route(scores, self.top_k, self.balance, score="sigmoid",
                                     groups=self.groups, top_groups=self.top_groups, group_top=2,
                                     logit_scale=1 / 32, scale=1.0)
        offsets, order = bnn.bnn_group_rows(ids, self.experts)
        inner = bnn.bnn_experts_fc(bits, self.width, self.w0, offsets, order, self.thr0,
                                   self.flip0)
        routed = bnn.bnn_experts_sum(inner, self.hidden, self.w1, ids, weights, offsets, order,
                                     self.alpha1, dtype=torch.bfloat16)
        _, rows = bnn.bnn_group_rows(adapter, self.a.shape[0])
        shared = bnn.bnn_bgemm_lora(h, self.shared, adapter, self.a, self.b, self.adapter_scale,
                                    self.alpha, self.offset, order=rows)
        if details is not None:
            details.update(bits=bits, scores=scores, ids=ids, weights=weights, inner=inner,
                           routed=routed, shared=shared)
        return h + shared + routed


def main():
    rows = int(sys.argv[1]) if len(sys.argv) > 1 else 4096
    block = ExpertBlock()
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn((rows, block.width), generator=g, device="cuda").to(torch.bfloat16)
    adapter = torch.randint(-1, 16, (rows,), generator=g, device="cuda").to(torch.int32)
    out = block(h, adapter)
    torch.cuda.synchronize()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(20):
        out = block(h, adapter)
    end.record()
    torch.cuda.synchronize()
    print("%d rows: %.1f us per pass, output rms %.3f" % (
        rows, start.elapsed_time(end) / 20 * 1e3, out.float().square().mean().sqrt().item()))


if __name__ == "__main__":
    main()
