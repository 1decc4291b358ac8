"""Factors and counts given as tensors, which a program changes in place between
calls (a temperature, a number of alternatives): every call reads what they hold
then.  CPU only, in the manner of test_binding_streams."""
import ctypes

import torch

from paper_1808_00209_amd import bnn
from test_binding_streams import _t, lib  # noqa: F401


def _descs(lib, kind):  # noqa: F811
    return [ctypes.cast(args[0], ctypes.POINTER(kind)).contents for _, args in lib.calls]


def test_temperature(lib):  # noqa: F811
    z, t = _t(2, 100, dtype=torch.float32), torch.tensor(1.0)
    for value in (1.0, 0.25, 2.5):
        bnn.bnn_logprobs(z, _t(2), logit_scale=t.fill_(value))
    assert [d.logit_scale for d in _descs(lib, bnn.LogprobsDesc)] == [1.0, 0.25, 2.5]


def test_alternatives(lib):  # noqa: F811
    """Also what is allocated for them: the outputs and the workspace."""
    z, k = _t(2, 20000, dtype=torch.float32), torch.tensor(8)
    for value in (8, 3, 20):
        out = bnn.bnn_logprobs(z, top_k=k.fill_(value))
        assert out[2].shape == out[3].shape == (2, value)
    got = _descs(lib, bnn.LogprobsDesc)
    assert [d.top_k for d in got] == [8, 3, 20]
    assert [args[-2] for _, args in lib.calls] == [bnn.bnn_logprobs_workspace_size(d) for d in got]


def test_eps(lib):  # noqa: F811
    x, eps = _t(3, 64, dtype=torch.bfloat16), torch.tensor(0.5)
    for value in (0.5, 0.125):
        bnn.bnn_rmsnorm(x, eps=eps.fill_(value))
    assert [d.eps for d in _descs(lib, bnn.RmsnormDesc)] == [0.5, 0.125]


def test_groups(lib):  # noqa: F811
    ids, G = _t(70000), torch.tensor(900)
    for value in (5, 900, 64):
        offsets, _ = bnn.bnn_group_rows(ids, G.fill_(value))
        assert offsets.shape == (value + 1,)
    assert [args[1] for _, args in lib.calls] == [5, 900, 64]
    assert [args[-2] for _, args in lib.calls] == [bnn.bnn_group_rows_workspace_size(70000, g)
                                                   for g in (5, 900, 64)]


def test_nothing_is_kept_alive(lib):  # noqa: F811
    import gc
    import weakref
    t = torch.tensor(1.0)
    gone = weakref.ref(t)
    bnn.bnn_logprobs(_t(2, 100, dtype=torch.float32), _t(2), logit_scale=t)
    del t
    gc.collect()
    assert gone() is None
