"""A call on a stream of the caller's (stream=s): what the binding allocates for
it is memory of that stream, so that the allocator hands it to no other work
before the call's kernels are done; an output, which the caller may use on the
current stream, is held for that one too.  CPU only: host tensors that say they
are on the device, and a library that launches nothing."""
import contextlib
import types

import pytest
import torch

from paper_1808_00209_amd import bnn

CURRENT = types.SimpleNamespace(cuda_stream=0x10, name="current")
OTHER = types.SimpleNamespace(cuda_stream=0x20, name="other")


class Device(torch.Tensor):
    """A host tensor that passes for one on the device and knows the stream it
    was made on (`on`) and those it was recorded on (`held`)."""
    is_cuda = True

    def new_empty(self, *size, **kw):
        return _made(torch.empty(*size, **kw))

    def zero_(self):
        _zeroed.append(_streams[-1].name)
        return super().zero_()

    def record_stream(self, stream):
        self.held.append(stream.name)


_streams = [CURRENT]
_allocated, _zeroed = [], []


def _made(t):
    t = t.as_subclass(Device)
    t.on, t.held = _streams[-1].name, []
    _allocated.append(t)
    return t


class Library:
    """Sizes come from the real library; every other call is noted."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith(("_size", "_dims")) or name == "bnn_last_error":
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return bnn.BNN_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    @contextlib.contextmanager
    def on(stream):
        _streams.append(stream)
        yield
        _streams.pop()

    fake = Library(bnn.load())
    monkeypatch.setattr(bnn, "load", lambda: fake)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _streams[-1])
    monkeypatch.setattr(torch, "empty", _host_empty)
    _allocated.clear()
    _zeroed.clear()
    return fake


_torch_empty = torch.empty


def _host_empty(*size, device=None, **kw):
    t = _torch_empty(*size, **kw)
    return t if device is None else _made(t)


def _t(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(Device)


def _route(**kw):
    bnn.bnn_route(_t(4, 8, dtype=torch.float32), 2, **kw)


def _group(**kw):
    bnn.bnn_group_rows(_t(20000), 5, **kw)


def _experts_fc(**kw):
    bnn.bnn_experts_fc(_t(6, 2), 64, _t(3, 40, 2), _t(4), _t(12), _t(3, 40), **kw)


def _experts_sum(**kw):
    T, N, K = 3000, 1000, 100
    bnn.bnn_experts_sum(_t(T, 4), K, _t(3, N, 4), _t(T, 2), _t(T, 2, dtype=torch.float32), _t(4),
                        _t(2 * T), **kw)


def _lora(**kw):
    f = torch.float32
    bnn.bnn_bgemm_lora(_t(50, 64, dtype=f), _t(40, 2), _t(50), _t(2, 8, 64, dtype=f),
                       _t(2, 40, 8, dtype=f), **kw)


def _conv(**kw):
    bnn.bnn_bconv2d(bnn.conv_desc(1, 8, 8, 32, 32), _t(64), _t(9, 32), **kw)


def _conv_prepared(**kw):
    bnn.bnn_bconv2d_prepared(bnn.conv_desc(1, 8, 8, 32, 32), _t(64), _t(9, 32),
                             _t(8, dtype=torch.uint8), **kw)


def _prepare(**kw):
    bnn.bnn_prepare_weights(_t(64, 3, 3, 2), 64, 3, 3, 64, **kw)


def _first(**kw):
    bnn.bnn_fconv2d_binw(bnn.conv_desc(1, 8, 8, 3, 32), _t(192, dtype=torch.float32), _t(9, 32), **kw)


def _conv_input(**kw):
    bnn.bnn_bconv2d_input(bnn.conv_desc(1, 8, 8, 3, 32), bnn.INPUT_THRESHOLD,
                          _t(192, dtype=torch.float32), None, _t(9, 32), **kw)


def _pair_desc():
    return bnn.conv_desc(1, 8, 8, 3, 32), bnn.conv_desc(1, 8, 8, 32, 32)


def _first_pair(**kw):
    bnn.bnn_fconv_bconv2d(*_pair_desc(), _t(192, dtype=torch.float32), _t(288), _t(32), None, _t(288),
                          _t(32), **kw)


def _input_pair(**kw):
    bnn.bnn_input_bconv_bconv2d(*_pair_desc(), bnn.INPUT_THRESHOLD, _t(192, dtype=torch.float32),
                                None, _t(288), _t(32), None, _t(288), _t(32), **kw)


def _conv_pair(**kw):
    bnn.bnn_bconv_bconv2d(*_pair_desc(), _t(64), _t(288), _t(32), None, _t(288), _t(32), **kw)


def _binarize(**kw):
    bnn.bnn_binarize_input(bnn.INPUT_THRESHOLD, _t(1, 8, 8, 3, dtype=torch.float32), **kw)


def _pack(**kw):
    bnn.bnn_pack_bits(_t(5, 40, dtype=torch.float32), **kw)


def _fc(**kw):
    bnn.bnn_bgemm(_t(4, 2), _t(40, 2), 64, **kw)


def _fc_pair(**kw):
    bnn.bnn_bfc_pair(_t(4, 2), 64, _t(40, 2), _t(40), None, _t(8, 2), 8, **kw)


def _fc_tail(**kw):
    bnn.bnn_bfc_tail(_t(4, 2), 64, _t(40, 2), _t(40), None, _t(8, 2), 8, _t(8), **kw)


def _net():
    return bnn.Network([dict(kind=bnn.LAYER_INPUT_THRESHOLD, C=32, offset=_t(32, dtype=torch.float32)),
                        dict(kind=bnn.LAYER_BFC_LOGITS, K=64 * 32, N=4, w=_t(4, 64))],
                       8, 8, 32)


def _forward(**kw):
    bnn.bnn_forward(_net(), _t(2, 8, 8, 32, dtype=torch.float32), **kw)


def _forward_noalloc(**kw):
    bnn.bnn_forward_noalloc(_net(), _t(2, 8, 8, 32, dtype=torch.float32), **kw)


CALLS = {  # outputs, workspaces
    _route: (2, 0), _group: (2, 1), _experts_fc: (1, 0), _experts_sum: (1, 1), _lora: (1, 1),
    _conv: (2, 0), _conv_prepared: (2, 0), _prepare: (1, 0), _first: (2, 0), _conv_input: (2, 0),
    _first_pair: (1, 0), _input_pair: (1, 0), _conv_pair: (1, 0), _binarize: (1, 0), _pack: (1, 0),
    _fc: (2, 0), _fc_pair: (1, 0), _fc_tail: (1, 0), _forward: (1, 1), _forward_noalloc: (1, 0),
}


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__[1:])
def test_memory_of_the_stream_that_the_call_runs_on(lib, call):
    outputs, workspaces = CALLS[call]
    call(stream=OTHER)
    assert len(_allocated) == outputs + workspaces
    assert {t.on for t in _allocated} == {"other"}
    held = [t.held for t in _allocated]
    assert held.count(["current"]) == outputs and held.count([]) == workspaces
    assert _zeroed == ["other"] * (call is _forward)  # its accumulators
    (_, args), = lib.calls
    assert args[-1] == OTHER.cuda_stream


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__[1:])
def test_memory_of_the_current_stream_without_one(lib, call):
    call()
    assert len(_allocated) == sum(CALLS[call])
    assert {t.on for t in _allocated} == {"current"} and not any(t.held for t in _allocated)
    (_, args), = lib.calls
    assert args[-1] == CURRENT.cuda_stream
