"""The calls of tests/test_gpu_expert_block.py one after another at sizes that
take the kernels of many rows (tests/test_expert_forms.py shows it): every step
against its definition, on the matrix cores and on the vector kernels, and as a
graph."""
import pytest
import torch

import test_gpu_expert_block as small
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

ROWS = [5000, 33000]
EXPERTS, TOP_K = 16, 4  # of the block


@pytest.mark.parametrize("algo", [bnn.ALGO_AUTO, bnn.ALGO_VALU], ids=["matrix", "vector"])
def test_every_step_against_its_definition(algo):
    block = small._block()
    assert (block.experts, block.top_k) == (EXPERTS, TOP_K)
    with bnn.options(algo=algo):
        small.test_every_step_against_its_definition(ROWS[0])


@pytest.mark.parametrize("T", ROWS)
def test_as_a_graph(T):
    small.test_as_a_graph(T)


@pytest.mark.parametrize("T", ROWS)
def test_twice_and_on_a_stream_of_its_own(T):
    block = small._block()
    h, adapter = small._inputs(T, 2)
    want = {}
    out = block(h, adapter, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            got = {}
            again = block(h, adapter, got)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    for k in want:
        assert torch.equal(want[k], got[k]), k
