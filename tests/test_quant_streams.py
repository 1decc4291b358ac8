"""The norm, the 8-bit product and the log probabilities on a stream of the
caller's: what they allocate is memory of that stream, and outputs are held for
the current one too.  CPU only, in the manner of test_binding_streams."""
import pytest
import torch

from paper_1808_00209_amd import bnn
from test_binding_streams import OTHER, _allocated, _t, lib  # noqa: F401


def _norm(D):
    f = torch.bfloat16
    return lambda **kw: bnn.bnn_rmsnorm(_t(5, D, dtype=f), _t(D, dtype=f), _t(5, D, dtype=f), want_y=True, **kw)


def _q8(**kw):
    b = torch.int8
    bnn.bnn_q8gemm(_t(5, 64, dtype=b), _t(7, 64, dtype=b), _t(5, dtype=torch.float32), **kw)


def _logprobs(**kw):
    bnn.bnn_logprobs(_t(2, 20000, dtype=torch.float32), _t(2, 3), 4, **kw)


@pytest.mark.parametrize("call, outputs, scratch", [
    (_norm(64), 4, 0), (_norm(33), 4, 0), (_q8, 1, 0), (_logprobs, 4, 1)])
def test_memory_of_a_call(lib, call, outputs, scratch):  # noqa: F811
    call()
    assert [t.on for t in _allocated] == ["current"] * (outputs + scratch)
    _allocated.clear()
    call(stream=OTHER)
    assert [t.on for t in _allocated] == ["other"] * (outputs + scratch)
    assert sorted(len(t.held) for t in _allocated) == [0] * scratch + [1] * outputs
    assert all(t.held in ([], ["current"]) for t in _allocated)
    assert [args[-1] for _, args in lib.calls] == [0x10, 0x20]
