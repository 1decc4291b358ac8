"""Refusals of the mixture-of-experts calls: every bad argument gives its
status and text before anything is launched (CPU only: the pointers are never
read), the sizes of the workspaces, and the binding's own checks."""
import ctypes

import pytest
import torch

import experts_ref as ref
from paper_1808_00209_amd import bnn

P = 0x1000  # a non-NULL, 16-byte aligned pointer that is never read


@pytest.fixture(scope="module")
def lib():
    return bnn.load()


def _refused(status, want, text):
    assert bnn.STATUS_NAMES[status] == want
    assert text in bnn.last_error()


def _route_desc(**kw):
    f = dict(E=64, top_k=8, groups=1, top_groups=1, group_top=1, score=0, renorm=1, dtype=0,
             scale=1.0, logit_scale=1.0)
    f.update(kw)
    return bnn.RouteDesc(**f)


@pytest.mark.parametrize("kw, text", [
    (dict(E=0), "experts"), (dict(E=1025), "experts"), (dict(top_k=0), "top_k"),
    (dict(top_k=17), "top_k"), (dict(E=4, top_k=5), "top_k"), (dict(groups=0), "groups"),
    (dict(groups=7), "groups"), (dict(E=1000, groups=125), "groups"),
    (dict(groups=8, top_groups=9), "top_groups"), (dict(top_groups=0), "top_groups"),
    (dict(group_top=3), "group_top"), (dict(score=2), "score"), (dict(renorm=2), "renorm"),
    (dict(dtype=4), "dtype"), (dict(logit_scale=0.0), "logit_scale"),
    (dict(logit_scale=float("inf")), "logit_scale"), (dict(scale=float("nan")), "scale")])
def test_route_descriptor(lib, kw, text):
    d = _route_desc(**kw)
    _refused(lib.bnn_route(ctypes.byref(d), 1, P, 2048, None, P, P, None), "BNN_ERR_SHAPE", text)


def test_route_arguments(lib):
    d = _route_desc()
    call = lambda T=1, x=P, s=64, i=P, w=P: lib.bnn_route(ctypes.byref(d), T, x, s, None, i, w, None)  # noqa: E731
    for kw in (dict(x=None), dict(i=None), dict(w=None)):
        _refused(call(**kw), "BNN_ERR_NULL", "non-NULL")
    _refused(lib.bnn_route(None, 1, P, 64, None, P, P, None), "BNN_ERR_NULL", "descriptor")
    _refused(call(s=63), "BNN_ERR_SHAPE", "stride")
    _refused(call(T=-1), "BNN_ERR_SHAPE", "T=-1")
    _refused(call(T=1 << 24), "BNN_ERR_SHAPE", "T=")
    _refused(call(x=P + 2), "BNN_ERR_SHAPE", "aligned")
    assert call(T=0, x=None, i=None, w=None) == bnn.BNN_OK


def test_group_rows_arguments(lib):
    def call(M=4, G=2, i=P, f=P, o=P, ws=P, n=1 << 40):
        return lib.bnn_group_rows(M, G, i, f, o, ws, n, None)

    n = ctypes.c_size_t()
    for kw in (dict(M=-1), dict(M=1 << 24), dict(G=0), dict(G=1025)):
        _refused(call(**kw), "BNN_ERR_SHAPE", "group_rows")
        size = dict(M=4, G=2)
        size.update(kw)
        _refused(lib.bnn_group_rows_workspace_size(size["M"], size["G"], ctypes.byref(n)),
                 "BNN_ERR_SHAPE", "group_rows")
    for kw in (dict(i=None), dict(f=None), dict(o=None), dict(M=0, f=None)):
        _refused(call(**kw), "BNN_ERR_NULL", "group_rows")
    _refused(lib.bnn_group_rows_workspace_size(4, 2, None), "BNN_ERR_NULL", "bytes")
    assert bnn.bnn_group_rows_workspace_size(1000, 64) == 0
    need = bnn.bnn_group_rows_workspace_size(1 << 20, 64)
    _refused(call(M=1 << 20, G=64, n=need - 1), "BNN_ERR_WORKSPACE", "group_rows")
    _refused(call(M=1 << 20, G=64, ws=None), "BNN_ERR_WORKSPACE", "group_rows")
    _refused(call(M=1 << 20, G=64, ws=P + 4), "BNN_ERR_ALIGN", "group_rows")


def _experts_desc(**kw):
    f = dict(T=4, top_k=2, E=3, N=40, K=70, share=1)
    f.update(kw)
    return bnn.ExpertsDesc(**f)


BAD_EXPERTS = [dict(E=0), dict(E=1025), dict(top_k=0), dict(top_k=17), dict(N=0), dict(K=0),
               dict(N=65537), dict(K=65536), dict(share=2), dict(T=-1), dict(T=1 << 23),
               dict(T=1 << 20, N=65536)]


@pytest.mark.parametrize("kw", BAD_EXPERTS, ids=str)
def test_experts_descriptor(lib, kw):
    d, n = _experts_desc(**kw), ctypes.c_size_t()
    _refused(lib.bnn_experts_fc(ctypes.byref(d), P, P, P, P, P, None, P, None), "BNN_ERR_SHAPE",
             "experts_fc")
    _refused(lib.bnn_experts_sum(ctypes.byref(d), P, P, P, P, P, P, None, 0, P, P, 1 << 40, None),
             "BNN_ERR_SHAPE", "experts_sum")
    _refused(lib.bnn_experts_sum_workspace_size(ctypes.byref(d), ctypes.byref(n)),
             "BNN_ERR_SHAPE", "experts_sum")


def test_experts_pointers(lib):
    d = ctypes.byref(_experts_desc())
    good = [P] * 5 + [None, P]  # x w offsets order thr flip out
    for i in (0, 1, 2, 3, 4, 6):
        a = list(good)
        a[i] = None
        _refused(lib.bnn_experts_fc(d, *a, None), "BNN_ERR_NULL", "experts_fc")
    for i in (0, 1, 6):
        a = list(good)
        a[i] = P + 4
        _refused(lib.bnn_experts_fc(d, *a, None), "BNN_ERR_ALIGN", "experts_fc")
    _refused(lib.bnn_experts_fc(None, *good, None), "BNN_ERR_NULL", "descriptor")
    good = [P] * 6 + [None, 0, P, P, 1 << 40]  # x w ids weights offsets order alpha dtype y ws n
    for i in (0, 1, 2, 3, 4, 5, 8):
        a = list(good)
        a[i] = None
        _refused(lib.bnn_experts_sum(d, *a, None), "BNN_ERR_NULL", "experts_sum")
    for i in (0, 1, 8):
        a = list(good)
        a[i] = P + 4
        _refused(lib.bnn_experts_sum(d, *a, None), "BNN_ERR_ALIGN", "experts_sum")
    for t in (3, 4, -1):
        a = list(good)
        a[7] = t
        _refused(lib.bnn_experts_sum(d, *a, None), "BNN_ERR_SHAPE", "dtype")
    none = ctypes.byref(_experts_desc(T=0))
    assert lib.bnn_experts_fc(none, *[None] * 7, None) == bnn.BNN_OK
    assert lib.bnn_experts_sum(none, *[None] * 7, 0, None, None, 0, None) == bnn.BNN_OK


def _lora_desc(**kw):
    f = dict(M=5, N=40, K=70, adapters=3, rank=8, dtype=2, out_dtype=2)
    f.update(kw)
    return bnn.LoraDesc(**f)


@pytest.mark.parametrize("kw, status", [
    (dict(M=-1), "SHAPE"), (dict(M=1 << 24), "SHAPE"), (dict(N=0), "SHAPE"), (dict(N=65537), "SHAPE"),
    (dict(K=0), "SHAPE"), (dict(K=65537), "SHAPE"), (dict(adapters=0), "SHAPE"),
    (dict(adapters=1025), "SHAPE"), (dict(rank=0), "SHAPE"), (dict(rank=12), "UNSUPPORTED"),
    (dict(M=1 << 22, N=65536), "SHAPE"), (dict(rank=264), "UNSUPPORTED"), (dict(dtype=3), "SHAPE"), (dict(out_dtype=3), "SHAPE")], ids=str)
def test_lora_descriptor(lib, kw, status):
    d, n = _lora_desc(**kw), ctypes.c_size_t()
    _refused(lib.bnn_bgemm_lora(ctypes.byref(d), P, 1 << 20, None, P, None, P, P, P, None, None, P, P,
                                1 << 50, None), "BNN_ERR_" + status, "lora")
    _refused(lib.bnn_bgemm_lora_workspace_size(ctypes.byref(d), ctypes.byref(n)),
             "BNN_ERR_" + status, "lora")


def test_lora_pointers_and_workspace(lib):
    d, n = ctypes.byref(_lora_desc()), ctypes.c_size_t()
    assert lib.bnn_bgemm_lora_workspace_size(d, ctypes.byref(n)) == bnn.BNN_OK
    # x stride offset w alpha ids a b scale order y ws bytes
    good = [P, 70, None, P, None, P, P, P, None, None, P, P, n.value]
    for i in (0, 3, 5, 6, 7, 10):
        a = list(good)
        a[i] = None
        _refused(lib.bnn_bgemm_lora(d, *a, None), "BNN_ERR_NULL", "lora")
    for i in (0, 3, 6, 7, 10, 11):
        a = list(good)
        a[i] = P + 8
        _refused(lib.bnn_bgemm_lora(d, *a, None), "BNN_ERR_ALIGN", "lora")
    a = list(good)
    a[1] = 69
    _refused(lib.bnn_bgemm_lora(d, *a, None), "BNN_ERR_SHAPE", "x_stride")
    a = list(good)
    a[12] = n.value - 1
    _refused(lib.bnn_bgemm_lora(d, *a, None), "BNN_ERR_WORKSPACE", "lora")
    a = list(good)
    a[11] = None
    _refused(lib.bnn_bgemm_lora(d, *a, None), "BNN_ERR_WORKSPACE", "lora")
    _refused(lib.bnn_bgemm_lora(None, *good, None), "BNN_ERR_NULL", "descriptor")
    _refused(lib.bnn_bgemm_lora_workspace_size(d, None), "BNN_ERR_NULL", "bytes")
    none = ctypes.byref(_lora_desc(M=0))
    assert lib.bnn_bgemm_lora(none, None, 70, *[None] * 10, 0, None) == bnn.BNN_OK


def test_workspace_sizes_grow_with_the_rows(lib):
    last = -1
    for M in (0, 1, 33, 4096):
        n = bnn.bnn_bgemm_lora_workspace_size(_lora_desc(M=M))
        assert n >= last
        last = n
    assert bnn.bnn_experts_sum_workspace_size(_experts_desc(T=0)) == 0


def test_the_binding_refuses_host_tensors_and_types():
    f, i = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int32)
    with pytest.raises(ValueError):
        bnn.bnn_route(f, 2)
    with pytest.raises(TypeError):
        bnn.bnn_route(f.double(), 2)
    with pytest.raises(TypeError):
        bnn.bnn_group_rows(i, 4)
    with pytest.raises(TypeError):
        bnn.bnn_experts_fc(i, 256, i, i, i, i)
    with pytest.raises(TypeError):
        bnn.bnn_experts_sum(i, 256, i, i, f, i, i)
    with pytest.raises(TypeError):
        bnn.bnn_bgemm_lora(i, i, i, f, f)


def test_the_reference_on_closed_forms():
    """The 64-bit definitions that the kernels are compared with."""
    ids, w, _ = ref.route([[0.0, 1.0, 1.0, float("-inf")]], 4, renorm=False)
    e = 2.718281828459045
    assert ids.tolist() == [[1, 2, 0, -1]]
    assert w[0] == pytest.approx([e / (1 + 2 * e)] * 2 + [1 / (1 + 2 * e), 0], abs=1e-12)
    off, order = ref.group_rows([1, -1, 0, 1, 7], 2)
    assert off.tolist() == [0, 1, 3] and order.tolist() == [2, 0, 3, 1, 4]
    assert ref.pm1([[-0x80000000, 1]], 64)[0, [0, 1, 63]].tolist() == [1, -1, 1]
    assert ref.pack([[1, 0, 1]]).view("uint32").tolist() == [[0xA0000000]]
    x, wt = ref.pack([[1, 1, 1, 0]]), ref.pack([[[1, 1, 0, 1]]])
    assert ref.expert_sums(x, wt, [0, -1], 4).tolist() == [[0], [0]]
    assert ref.experts_fc(x, wt, [0], 4, [[0]]).view("uint32").tolist() == [[0x80000000]]
    assert ref.experts_fc(x, wt, [0], 4, [[1]]).tolist() == [[0]]
