"""Refusals of the 8-bit layers' and the log probabilities' calls: every bad
argument gives its status and text before anything is launched (CPU only: the
pointers are never read), and the binding's own checks."""
import ctypes
import types

import pytest
import torch

from paper_1808_00209_amd import bnn

P = 0x1000  # a non-NULL, 16-byte aligned pointer that is never read


@pytest.fixture(scope="module")
def lib():
    return bnn.load()


def _refused(status, want, text):
    assert bnn.STATUS_NAMES[status] == want
    assert text in bnn.last_error()


def _norm(lib, x=P, xs=64, r=P, rs=64, w=P, h=P, y=P + 64, q=P, qs=64, s=P, **kw):
    d = dict(M=4, D=64, dtype=2, weight_dtype=2, eps=1e-6)
    d.update(kw)
    return lib.bnn_rmsnorm(ctypes.byref(bnn.RmsnormDesc(**d)), x, xs, r, rs, w, h, y, q, qs, s, None)


@pytest.mark.parametrize("kw, status, text", [
    (dict(M=-1), "SHAPE", "M=-1"), (dict(M=1 << 24), "SHAPE", "M="), (dict(D=0), "SHAPE", "D=0"),
    (dict(D=65537, xs=65537, rs=65537, qs=65537), "SHAPE", "D="), (dict(dtype=3), "SHAPE", "dtype"),
    (dict(dtype=-1), "SHAPE", "dtype"), (dict(weight_dtype=1), "SHAPE", "weight_dtype"),
    (dict(weight_dtype=3), "SHAPE", "weight_dtype"), (dict(eps=-1e-9), "SHAPE", "eps"),
    (dict(eps=float("nan")), "SHAPE", "eps"), (dict(eps=float("inf")), "SHAPE", "eps"),
    (dict(xs=63), "SHAPE", "stride"), (dict(rs=63), "SHAPE", "stride"), (dict(qs=63), "SHAPE", "stride"),
    (dict(xs=(1 << 31) + 1), "SHAPE", "stride"), (dict(x=None), "NULL", "x must"),
    (dict(h=None, y=None, q=None, s=None), "NULL", "one of"), (dict(s=None), "NULL", "together"),
    (dict(q=None), "NULL", "together"), (dict(y=P), "SHAPE", "same rows"), (dict(x=P + 1), "SHAPE", "aligned"),
    (dict(r=P + 1), "SHAPE", "aligned"), (dict(h=P + 1), "SHAPE", "aligned"), (dict(y=P + 3), "SHAPE", "aligned"),
    (dict(w=P + 1), "SHAPE", "aligned"), (dict(weight_dtype=0, w=P + 2), "SHAPE", "aligned"),
    (dict(s=P + 2), "SHAPE", "aligned"), (dict(x=P, h=P, xs=80), "SHAPE", "in place"),
    (dict(r=P + 64, y=P + 64, rs=80), "SHAPE", "in place")])
def test_norm(lib, kw, status, text):
    _refused(_norm(lib, **kw), "BNN_ERR_" + status, text)


def test_norm_without_rows(lib):
    assert _norm(lib, M=0, x=None, r=None, h=None, y=None, q=None, s=None) == bnn.BNN_OK
    _refused(lib.bnn_rmsnorm(None, P, 1, None, 0, None, P, None, None, 0, None, None), "BNN_ERR_NULL", "descriptor")


def _q8(lib, x=P, xs=64, sx=P, w=P, ws=64, sw=P, b=P, y=P, **kw):
    d = dict(M=4, N=8, K=64, dtype=2)
    d.update(kw)
    return lib.bnn_q8gemm(ctypes.byref(bnn.Q8gemmDesc(**d)), x, xs, sx, w, ws, sw, b, y, None)


@pytest.mark.parametrize("kw, status, text", [
    (dict(M=-1), "SHAPE", "M=-1"), (dict(M=1 << 24), "SHAPE", "M="), (dict(N=0), "SHAPE", "N=0"),
    (dict(N=(1 << 20) + 1), "SHAPE", "N="), (dict(K=0), "SHAPE", "K=0"),
    (dict(K=131072, xs=131072, ws=131072), "SHAPE", "K="), (dict(M=1 << 23, N=1 << 13), "SHAPE", "too large"),
    (dict(dtype=3), "SHAPE", "dtype"), (dict(xs=63), "SHAPE", "stride"), (dict(ws=63), "SHAPE", "stride"),
    (dict(xs=(1 << 31) + 1), "SHAPE", "stride"), (dict(ws=(1 << 31) + 1), "SHAPE", "stride"),
    (dict(x=None), "NULL", "non-NULL"), (dict(w=None), "NULL", "non-NULL"), (dict(y=None), "NULL", "non-NULL"),
    (dict(y=P + 8), "ALIGN", "16-byte"), (dict(sx=P + 1), "SHAPE", "aligned"), (dict(sw=P + 2), "SHAPE", "aligned"),
    (dict(b=P + 3), "SHAPE", "aligned")])
def test_q8gemm(lib, kw, status, text):
    _refused(_q8(lib, **kw), "BNN_ERR_" + status, text)


def test_q8gemm_without_rows(lib):
    assert _q8(lib, M=0, x=None, y=None) == bnn.BNN_OK
    _refused(lib.bnn_q8gemm(None, P, 1, None, P, 1, None, None, P, None), "BNN_ERR_NULL", "descriptor")


def _lp(lib, x=P, stride=30000, i=P, lp=P, e=P, ti=P, tl=P, ws=P, n_ws=1 << 40, **kw):
    d = dict(T=4, V=30000, n=2, top_k=5, dtype=0, logit_scale=1.0)
    d.update(kw)
    return lib.bnn_logprobs(ctypes.byref(bnn.LogprobsDesc(**d)), x, stride, i, lp, e, ti, tl, ws, n_ws, None)


@pytest.mark.parametrize("kw, status, text", [
    (dict(T=-1), "SHAPE", "T=-1"), (dict(T=1 << 24), "SHAPE", "T="), (dict(V=0), "SHAPE", "V=0"),
    (dict(V=(1 << 24) + 1, stride=1 << 25), "SHAPE", "V="), (dict(n=-1), "SHAPE", "n=-1"),
    (dict(n=1025), "SHAPE", "n="), (dict(top_k=-1), "SHAPE", "top_k"), (dict(top_k=33), "SHAPE", "top_k"),
    (dict(V=4, top_k=5), "SHAPE", "top_k"), (dict(dtype=4), "SHAPE", "dtype"), (dict(dtype=-1), "SHAPE", "dtype"),
    (dict(logit_scale=0.0), "SHAPE", "logit_scale"), (dict(logit_scale=-1.0), "SHAPE", "logit_scale"),
    (dict(logit_scale=2.0 ** 101), "SHAPE", "logit_scale"),
    (dict(logit_scale=float("nan")), "SHAPE", "logit_scale"), (dict(logit_scale=float("inf")), "SHAPE", "logit_scale"),
    (dict(stride=29999), "SHAPE", "stride"), (dict(stride=(1 << 31) + 1), "SHAPE", "stride"),
    (dict(x=None), "NULL", "logits"), (dict(i=None), "NULL", "ids"), (dict(lp=None), "NULL", "logp"),
    (dict(ti=None), "NULL", "top_ids"), (dict(tl=None), "NULL", "top_logp"),
    (dict(n=0, top_k=0, e=None), "NULL", "nothing"), (dict(x=P + 2), "SHAPE", "aligned"),
    (dict(i=P + 2), "SHAPE", "aligned"), (dict(lp=P + 1), "SHAPE", "aligned"), (dict(e=P + 1), "SHAPE", "aligned"),
    (dict(ti=P + 2), "SHAPE", "aligned"), (dict(tl=P + 2), "SHAPE", "aligned"),
    (dict(n_ws=16), "WORKSPACE", "needed"), (dict(ws=None), "WORKSPACE", "needed"), (dict(ws=P + 8), "ALIGN", "workspace")])
def test_logprobs(lib, kw, status, text):
    _refused(_lp(lib, **kw), "BNN_ERR_" + status, text)


def test_logprobs_workspace(lib):
    n = ctypes.c_size_t()
    size = lambda T, V, k: bnn.bnn_logprobs_workspace_size(bnn.LogprobsDesc(T, V, 1, k, 0, 1.0))  # noqa: E731
    assert _lp(lib, T=0, x=None, i=None, ws=None, n_ws=0) == bnn.BNN_OK
    _refused(lib.bnn_logprobs(None, P, 1, P, P, P, P, P, P, 0, None), "BNN_ERR_NULL", "descriptor")
    _refused(lib.bnn_logprobs_workspace_size(None, ctypes.byref(n)), "BNN_ERR_NULL", "descriptor")
    d = bnn.LogprobsDesc(4, 8, 1, 9, 0, 1.0)
    _refused(lib.bnn_logprobs_workspace_size(ctypes.byref(d), ctypes.byref(n)), "BNN_ERR_SHAPE", "top_k")
    _refused(lib.bnn_logprobs_workspace_size(ctypes.byref(bnn.LogprobsDesc(4, 8, 1, 2, 0, 1.0)), None),
             "BNN_ERR_NULL", "bytes")
    assert size(5, 700, 8) == 0
    for V in (5000, 50000, 1 << 24):
        sizes = [size(T, V, 20) for T in (0, 1, 2, 3, 10, 100, 1000, 1023, 1024, 1025, 9999, (1 << 24) - 1)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[-1] < 1 << 20


class Device(torch.Tensor):
    """A host tensor that passes for one on the device."""
    is_cuda = True


def _made(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


def test_binding_checks():
    """Wrong types, shapes and rows, before the library is called."""
    x, q, i32 = _made(4, 8), _made(4, 8, dtype=torch.int8), torch.int32
    for error, call in [
            (TypeError, lambda: bnn.bnn_rmsnorm(_made(4, 8, dtype=torch.float64))),
            (ValueError, lambda: bnn.bnn_rmsnorm(torch.zeros(4, 8))),
            (ValueError, lambda: bnn.bnn_rmsnorm(_made(8))),
            (ValueError, lambda: bnn.bnn_rmsnorm(_made(8, 4).t())),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, _made(7))),
            (TypeError, lambda: bnn.bnn_rmsnorm(x, _made(8, dtype=torch.float16))),
            (TypeError, lambda: bnn.bnn_rmsnorm(x, None, _made(4, 8, dtype=torch.bfloat16))),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, None, _made(4, 9))),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, sum=_made(3, 8))),
            (TypeError, lambda: bnn.bnn_rmsnorm(x, y=_made(4, 8, dtype=torch.float16))),
            (TypeError, lambda: bnn.bnn_rmsnorm(x, q=_made(4, 8))),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, q=_made(4, 9, dtype=torch.int8))),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, scale=_made(5))),
            (ValueError, lambda: bnn.bnn_rmsnorm(x, want_q=False, want_y=True, scale=_made(4))),
            (TypeError, lambda: bnn.bnn_q8gemm(x, q)), (TypeError, lambda: bnn.bnn_q8gemm(q, x)),
            (ValueError, lambda: bnn.bnn_q8gemm(q, _made(4, 9, dtype=torch.int8))),
            (ValueError, lambda: bnn.bnn_q8gemm(q, _made(8, dtype=torch.int8))),
            (ValueError, lambda: bnn.bnn_q8gemm(q, q, _made(3))), (ValueError, lambda: bnn.bnn_q8gemm(q, q, None, _made(3))),
            (ValueError, lambda: bnn.bnn_q8gemm(q, q, bias=_made(3))),
            (TypeError, lambda: bnn.bnn_q8gemm(q, q, _made(4, dtype=torch.float16))),
            (TypeError, lambda: bnn.bnn_q8gemm(q, q, dtype=i32)),
            (ValueError, lambda: bnn.bnn_q8gemm(q, q, out=_made(4, 5))),
            (ValueError, lambda: bnn.bnn_q8gemm(q.as_strided((3, 8), (4, 1)), q)),
            (TypeError, lambda: bnn.bnn_logprobs(q)), (ValueError, lambda: bnn.bnn_logprobs(_made(8))),
            (TypeError, lambda: bnn.bnn_logprobs(x, _made(4, dtype=torch.int64))),
            (ValueError, lambda: bnn.bnn_logprobs(x, _made(3, dtype=i32))),
            (ValueError, lambda: bnn.bnn_logprobs(x, _made(4, 2, 2, dtype=i32))),
            (ValueError, lambda: bnn.bnn_logprobs(x, logp=_made(4))),
            (ValueError, lambda: bnn.bnn_logprobs(x, top_ids=_made(4, 2, dtype=i32))),
            (ValueError, lambda: bnn.bnn_logprobs(x, top_k=2, top_ids=_made(4, 3, dtype=i32))),
            (bnn.BnnError, lambda: bnn.bnn_logprobs(x, top_k=9)),
            (TypeError, lambda: bnn.bnn_logprobs(_made(4, 9000), top_k=2, workspace=_made(1 << 20)))]:
        with pytest.raises(error):
            call()


def test_tensors_of_one_device(monkeypatch):
    on = lambda i: types.SimpleNamespace(get_device=lambda: i, device="cuda:%d" % i)  # noqa: E731
    monkeypatch.setattr(bnn, "_raw_device", lambda: 1)
    bnn._together(on(1), None, on(1))
    with pytest.raises(ValueError, match="in one call"):
        bnn._together(on(1), None, on(0))
    with pytest.raises(ValueError, match="current device"):
        bnn._together(on(0), on(0))
