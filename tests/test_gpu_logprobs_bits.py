"""The last bits of almost certain answers, whose ln p and entropy are differences
of nearly equal numbers, where the certain one comes behind others in its wave's
share of the row.

A row has three answers of 0 and one of h = 5..10.9, all others out of reach:
four terms, so that the sums have three roundings (half a unit each) and the
largest term one exp2 (a unit); log2 has a unit of a result below 0.03.  In units
of fp32 at 1 that is 2^-23 + 3 * 2^-24 + 2^-24 at most: ln p within 6 * 2^-24.
The entropy adds sum p |ln p| of the three, which has 24 bits less what a few
steps lose: 2^-20 of itself."""
import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu


# rows of one wave, of four, of sixteen, in parts
@pytest.mark.parametrize("T, V, waves", [(2100, 4090, 1), (600, 17000, 4), (200, 12000, 4), (170, 50000, 16), (3, 140000, 4)])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "int32"])
def test_certain_answer_comes_late(T, V, waves, kind):
    g = torch.Generator().manual_seed(V)
    rounds = V // (1024 * waves)
    wave = torch.randint(0, waves, (T,), generator=g)
    z = torch.full((T, V), -2 ** 31 if kind == "int32" else -float("inf"), dtype=torch.float64)
    rows = torch.arange(T)
    for i in range(3):
        z[rows, 1024 * wave + 300 * i + torch.randint(0, 300, (T,), generator=g)] = 0
    last = torch.randint(1, rounds, (T,), generator=g) if rounds > 1 else torch.zeros(T, dtype=torch.long)
    at = 1024 * (waves * last + wave) + 901 + torch.randint(0, 100, (T,), generator=g)
    z[rows, at] = 5 + 5.9 * torch.rand(T, generator=g, dtype=torch.float64)
    scale = 1.0
    if kind == "int32":
        scale = 1 / 64
        z[rows, at] = (64 * z[rows, at]).round()
    z = z.to({"fp32": torch.float32, "bf16": torch.bfloat16, "int32": torch.int32}[kind])
    got = bnn.bnn_logprobs(z.cuda(), at.to(torch.int32).cuda(), logit_scale=scale)
    given, entropy, _, _ = ref.logprobs(z, at.to(torch.int32), 0, scale)
    off = (got[0].cpu().double() - given).abs().max().item()
    off_h = ((got[1].cpu().double() - entropy).abs() - 2.0 ** -20 * entropy).max().item()
    print("ln p off by %.2g, the entropy by %.2g" % (off, off_h))
    assert off <= 6 * 2.0 ** -24 and off_h <= 6 * 2.0 ** -24
