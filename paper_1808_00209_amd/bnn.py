"""ctypes binding of libbnn.so (C ABI in include/bnn.h).

Argument marshalling only: every function checks tensor dtypes, devices and
contiguity, allocates outputs with torch when the caller does not pass them,
and calls the C entry point of the same name on the current HIP stream, or on
the one given as ``stream``: what the call allocates is then memory of that
stream.  All computation happens in the library's HIP kernels.  Loading fails
loudly when libbnn.so has not been built
(``python -m paper_1808_00209_amd.build``).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbnn.so")

BNN_OK = 0
STATUS_NAMES = {0: "BNN_OK", 1: "BNN_ERR_NULL", 2: "BNN_ERR_SHAPE", 3: "BNN_ERR_ALIGN",
                4: "BNN_ERR_UNSUPPORTED", 5: "BNN_ERR_HIP", 6: "BNN_ERR_WORKSPACE"}

LAYER_INPUT_THRESHOLD = 1
LAYER_FCONV_BINW = 2
LAYER_BCONV = 3
LAYER_BFC = 4
LAYER_BFC_LOGITS = 5
LAYER_INPUT_GRAY = 6
LAYER_INPUT_LBP = 7
INPUT_THRESHOLD = 0
INPUT_GRAY = 1
INPUT_LBP = 2

# Every symbol include/bnn.h declares.
EXPORTED = ["bnn_last_error", "bnn_abi_version", "bnn_default_options", "bnn_set_options",
            "bnn_get_options", "bnn_pack_bits", "bnn_conv_output_dims",
            "bnn_bconv2d", "bnn_prepared_weights_size", "bnn_prepare_weights",
            "bnn_bconv2d_prepared", "bnn_fconv2d_binw", "bnn_binarize_input", "bnn_bconv2d_input",
            "bnn_fconv_bconv2d", "bnn_input_bconv_bconv2d", "bnn_bconv_bconv2d", "bnn_bfc_pair", "bnn_bfc_tail",
            "bnn_bgemm",
            "bnn_route", "bnn_group_rows_workspace_size", "bnn_group_rows", "bnn_experts_fc", "bnn_experts_sum_workspace_size",
            "bnn_experts_sum", "bnn_bgemm_lora_workspace_size", "bnn_bgemm_lora",
            "bnn_forward_workspace_size", "bnn_forward", "bnn_forward_noalloc"]

# Bytes of bnn_forward_noalloc's per-GPU scratch array (BNN_FORWARD_SCRATCH_BYTES).
FORWARD_SCRATCH_BYTES = 64 << 20
# Leading workspace bytes that must be zero before a workspace's first use
# (BNN_FORWARD_SYNC_BYTES: the FC tail kernel's accumulators, left zero by every call).
FORWARD_SYNC_BYTES = 69632


class BnnError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status


ALGO_AUTO = 0
ALGO_VALU = 1


class Options(ctypes.Structure):
    """bnn_options: the calling thread's kernel selection (never changes a result)."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("algo", "fuse_input", "fuse_first", "fc_chain", "conv1x1", "xcd_order",
                 "gemv_max_rows", "lds_weights", "late_thresholds", "fuse_pair")]


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("N", "H", "W", "C", "F", "KH", "KW", "stride", "pad", "pool")]


class Layer(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("C", ctypes.c_int32), ("F", ctypes.c_int32),
                ("KH", ctypes.c_int32), ("KW", ctypes.c_int32), ("stride", ctypes.c_int32),
                ("pad", ctypes.c_int32), ("pool", ctypes.c_int32), ("K", ctypes.c_int32),
                ("N", ctypes.c_int32), ("w", ctypes.c_void_p), ("thr", ctypes.c_void_p),
                ("flip", ctypes.c_void_p), ("offset", ctypes.c_void_p), ("wprep", ctypes.c_void_p)]


class RouteDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("E", "top_k", "groups", "top_groups", "group_top", "score", "renorm", "dtype")]
    _fields_ += [("scale", ctypes.c_float), ("logit_scale", ctypes.c_float)]


class ExpertsDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in
                                          ("top_k", "E", "N", "K", "share")]


class LoraDesc(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in
                                          ("N", "K", "adapters", "rank", "dtype", "out_dtype")]


_lib = None


def load(path: str = LIB_PATH):
    """Load libbnn.so and declare the C signatures (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libbnn.so not found at %s: build it with "
                           "`python -m paper_1808_00209_amd.build` (no fallback exists)" % path)
    lib = ctypes.CDLL(path)
    P, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.bnn_last_error.restype = ctypes.c_char_p
    lib.bnn_last_error.argtypes = []
    lib.bnn_abi_version.restype = i32
    lib.bnn_abi_version.argtypes = []
    lib.bnn_default_options.restype = None
    lib.bnn_default_options.argtypes = [ctypes.POINTER(Options)]
    lib.bnn_set_options.argtypes = [ctypes.POINTER(Options)]
    lib.bnn_get_options.argtypes = [ctypes.POINTER(Options)]
    lib.bnn_pack_bits.argtypes = [P, P, i64, i64, P, P]
    lib.bnn_conv_output_dims.argtypes = [ctypes.POINTER(ConvDesc)] + [ctypes.POINTER(i32)] * 4
    lib.bnn_bconv2d.argtypes = [ctypes.POINTER(ConvDesc), P, P, P, P, P, P, P]
    lib.bnn_prepared_weights_size.argtypes = [i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.bnn_prepare_weights.argtypes = [i32, i32, i32, i32, P, P, P]
    lib.bnn_bconv2d_prepared.argtypes = [ctypes.POINTER(ConvDesc), P, P, P, P, P, P, P, P]
    lib.bnn_fconv2d_binw.argtypes = [ctypes.POINTER(ConvDesc), P, P, P, P, P, P, P]
    lib.bnn_bgemm.argtypes = [i64, i64, i64, P, P, P, P, P, P, P]
    lib.bnn_binarize_input.argtypes = [i32, P, P, i32, i32, i32, i32, P, P]
    lib.bnn_bconv2d_input.argtypes = [ctypes.POINTER(ConvDesc), i32, P, P, P, P, P, P, P, P]
    lib.bnn_fconv_bconv2d.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvDesc),
                                      P, P, P, P, P, P, P, P, P, P]
    lib.bnn_input_bconv_bconv2d.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvDesc),
                                            i32, P, P, P, P, P, P, P, P, P, P, P]
    lib.bnn_bconv_bconv2d.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvDesc),
                                      P, P, P, P, P, P, P, P, P]
    lib.bnn_bfc_pair.argtypes = [i64, i64, i64, i64, P, P, P, P, P, P, P, P, P, P]
    lib.bnn_bfc_tail.argtypes = [i64, i64, i64, i64, P, P, P, P, P, P, P, P, P, P, P]
    lib.bnn_route.argtypes = [ctypes.POINTER(RouteDesc), i64, P, i64, P, P, P, P]
    lib.bnn_group_rows_workspace_size.argtypes = [i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.bnn_group_rows.argtypes = [i64, i32, P, P, P, P, ctypes.c_size_t, P]
    lib.bnn_experts_fc.argtypes = [ctypes.POINTER(ExpertsDesc), P, P, P, P, P, P, P, P]
    lib.bnn_experts_sum_workspace_size.argtypes = [ctypes.POINTER(ExpertsDesc),
                                                   ctypes.POINTER(ctypes.c_size_t)]
    lib.bnn_experts_sum.argtypes = [ctypes.POINTER(ExpertsDesc), P, P, P, P, P, P, P, i32, P, P,
                                    ctypes.c_size_t, P]
    lib.bnn_bgemm_lora_workspace_size.argtypes = [ctypes.POINTER(LoraDesc),
                                                  ctypes.POINTER(ctypes.c_size_t)]
    lib.bnn_bgemm_lora.argtypes = [ctypes.POINTER(LoraDesc), P, i64, P, P, P, P, P, P, P, P, P, P,
                                   ctypes.c_size_t, P]
    lib.bnn_forward_workspace_size.argtypes = [ctypes.POINTER(Layer), i32, i32, i32, i32, i32,
                                               ctypes.POINTER(ctypes.c_size_t)]
    lib.bnn_forward.argtypes = [ctypes.POINTER(Layer), i32, i32, i32, i32, i32, P, P,
                                ctypes.c_size_t, P, P]
    lib.bnn_forward_noalloc.argtypes = [ctypes.POINTER(Layer), i32, i32, i32, i32, i32, P, P, P]
    for name in EXPORTED:
        if name not in ("bnn_last_error", "bnn_abi_version", "bnn_default_options"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def last_error() -> str:
    return load().bnn_last_error().decode()


def _check(status: int):
    if status != BNN_OK:
        raise BnnError(status, last_error())


# A small layer's kernel takes 3-5 us, as long as it takes to get through this
# binding, so a call spends as little here as it can: pointers and the stream
# go to ctypes as plain ints, the stream handle comes without a Stream object
# around it, and a conv's output sizes are worked out here (host time of one
# call: a bgemm 9.9 -> 7.1 us, a small 3x3 conv 12.7 -> 9.3, a forward pass at
# one image 20.3 -> 19.2).
def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _dev(t, dtype, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or not t.is_cuda:
        raise TypeError("%s must be a CUDA(HIP) tensor of %s" % (name, dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


# A call's memory belongs to the stream that the call runs on (new_empty of a
# tensor on the current one): torch's allocator may hand the block to other work
# of that stream as soon as the tensor is dropped, and to no other's.
def _scratch(like, shape, dtype, stream):
    """A new tensor on like's device for the call alone."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _empty(like, shape, dtype, stream):
    """A new tensor on like's device that the caller gets, and may use and drop
    on the current stream."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    t = _scratch(like, shape, dtype, stream)
    t.record_stream(torch.cuda.current_stream(like.device))
    return t


def words(bits: int) -> int:
    return (bits + 31) // 32


def _u32(t):
    """torch has no uint32 arithmetic; packed words travel as int32 storage."""
    return _dev(t, torch.int32, "packed words")


# ---------------------------------------------------------------- options ---
def bnn_default_options() -> Options:
    o = Options()
    load().bnn_default_options(ctypes.byref(o))
    return o


def bnn_get_options() -> Options:
    o = Options()
    _check(load().bnn_get_options(ctypes.byref(o)))
    return o


def bnn_set_options(opt: Options = None, **fields) -> Options:
    """Set the calling thread's options: ``opt`` (default: the library
    defaults) with ``fields`` replaced.  Returns the options in force before."""
    prev = bnn_get_options()
    o = Options.from_buffer_copy(opt) if opt is not None else bnn_default_options()
    for k, v in fields.items():
        if k not in dict(Options._fields_):
            raise KeyError("unknown option %r" % k)
        setattr(o, k, int(v))
    _check(load().bnn_set_options(ctypes.byref(o)))
    return prev


@contextlib.contextmanager
def options(**fields):
    """``with bnn.options(algo=bnn.ALGO_VALU): ...`` -- the defaults with
    ``fields`` replaced, restored to what was in force on exit."""
    prev = bnn_set_options(None, **fields)
    try:
        yield
    finally:
        _check(load().bnn_set_options(ctypes.byref(prev)))


# ------------------------------------------------------------------ calls ---
def bnn_pack_bits(x, offset=None, out=None, stream=None):
    """Eq. (1)+(2): x [..., D] fp32 -> packed words [..., ceil(D/32)] (int32 storage)."""
    lib = load()
    x = _dev(x, torch.float32, "x")
    D = x.shape[-1]
    rows = x.numel() // D if D else 0
    if offset is not None:
        offset = _dev(offset, torch.float32, "offset")
    if out is None:
        out = _empty(x, tuple(x.shape[:-1]) + (words(D),), torch.int32, stream)
    _u32(out)
    _check(lib.bnn_pack_bits(_ptr(x), _ptr(offset), rows, D, _ptr(out), _stream(stream)))
    return out


def conv_desc(N, H, W, C, F, KH=3, KW=3, stride=1, pad=1, pool=0) -> ConvDesc:
    return ConvDesc(N, H, W, C, F, KH, KW, stride, pad, pool)


def bnn_conv_output_dims(desc: ConvDesc):
    lib = load()
    o = [ctypes.c_int32() for _ in range(4)]
    _check(lib.bnn_conv_output_dims(ctypes.byref(desc), *[ctypes.byref(v) for v in o]))
    return tuple(v.value for v in o)


def _output_dims(desc: ConvDesc):
    """bnn_conv_output_dims without the call for ordinary sizes; anything
    unusual goes through it, for its checks and messages."""
    H, W, KH, KW, pad, pool = desc.H, desc.W, desc.KH, desc.KW, desc.pad, desc.pool
    Ho, Wo = H + 2 * pad - KH + 1, W + 2 * pad - KW + 1
    if (0 < H < 32768 and 0 < W < 32768 and 0 < KH < 128 and 0 < KW < 128 and 0 <= pad < 128
            and Ho > 1 and Wo > 1 and desc.stride == 1 and 0 < desc.N and 0 < desc.C < 4096
            and 0 < desc.F < 16384 and desc.N * Ho * Wo < 1 << 24 and desc.N * H * W < 1 << 24
            and KH * KW * desc.C < 1 << 20):
        if pool == 2:
            return Ho, Wo, Ho // 2, Wo // 2
        if pool == 0:
            return Ho, Wo, Ho, Wo
    return bnn_conv_output_dims(desc)


def bnn_bconv2d(desc: ConvDesc, x, w, thr=None, flip=None, want_sums=True, want_bits=True,
                out_sums=None, out_bits=None, stream=None):
    """Binary conv (Eq. 3/4) with fused threshold/flip/OR-pool.  Returns
    (sums [N,Ho,Wo,F] int32 or None, bits [N,Hp,Wp,Fw] int32-storage or None)."""
    lib = load()
    Ho, Wo, Hp, Wp = _output_dims(desc)
    _u32(x)
    _u32(w)
    thr = _dev(thr, torch.int32, "thr")
    flip = _dev(flip, torch.int32, "flip")
    if want_sums and out_sums is None:
        out_sums = _empty(x, (desc.N, Ho, Wo, desc.F), torch.int32, stream)
    if want_bits and out_bits is None:
        out_bits = _empty(x, (desc.N, Hp, Wp, words(desc.F)), torch.int32, stream)
    _check(lib.bnn_bconv2d(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(thr), _ptr(flip),
                           _ptr(out_sums), _ptr(out_bits), _stream(stream)))
    return out_sums, out_bits


def bnn_prepared_weights_size(F, KH, KW, C) -> int:
    out = ctypes.c_size_t()
    _check(load().bnn_prepared_weights_size(F, KH, KW, C, ctypes.byref(out)))
    return out.value


def bnn_prepare_weights(w, F, KH, KW, C, out=None, stream=None):
    """Packed conv weights [F, KH, KW, ceil(C/32)] -> the matrix-core operand
    form (a uint8 device buffer of bnn_prepared_weights_size bytes)."""
    lib = load()
    _u32(w)
    if out is None:
        out = _empty(w, bnn_prepared_weights_size(F, KH, KW, C), torch.uint8, stream)
    _check(lib.bnn_prepare_weights(F, KH, KW, C, _ptr(w), _ptr(out), _stream(stream)))
    return out


def bnn_bconv2d_prepared(desc: ConvDesc, x, w, wprep, thr=None, flip=None, want_sums=True,
                         want_bits=True, out_sums=None, out_bits=None, stream=None):
    """bnn_bconv2d with prepared weights (wprep = bnn_prepare_weights of w)."""
    lib = load()
    Ho, Wo, Hp, Wp = _output_dims(desc)
    _u32(x)
    _u32(w)
    _dev(wprep, torch.uint8, "wprep")
    thr = _dev(thr, torch.int32, "thr")
    flip = _dev(flip, torch.int32, "flip")
    if want_sums and out_sums is None:
        out_sums = _empty(x, (desc.N, Ho, Wo, desc.F), torch.int32, stream)
    if want_bits and out_bits is None:
        out_bits = _empty(x, (desc.N, Hp, Wp, words(desc.F)), torch.int32, stream)
    _check(lib.bnn_bconv2d_prepared(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(wprep), _ptr(thr),
                                    _ptr(flip), _ptr(out_sums), _ptr(out_bits),
                                    _stream(stream)))
    return out_sums, out_bits


def bnn_fconv2d_binw(desc: ConvDesc, x, w, thr=None, flip=None, want_sums=True,
                     want_bits=True, out_sums=None, out_bits=None, stream=None):
    """fp32-input conv with packed +-1 weights; sums fp32 [N,Ho,Wo,F]."""
    lib = load()
    Ho, Wo, Hp, Wp = _output_dims(desc)
    _dev(x, torch.float32, "x")
    _u32(w)
    thr = _dev(thr, torch.int32, "thr")
    flip = _dev(flip, torch.int32, "flip")
    if want_sums and out_sums is None:
        out_sums = _empty(x, (desc.N, Ho, Wo, desc.F), torch.float32, stream)
    if want_bits and out_bits is None:
        out_bits = _empty(x, (desc.N, Hp, Wp, words(desc.F)), torch.int32, stream)
    _check(lib.bnn_fconv2d_binw(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(thr), _ptr(flip),
                                _ptr(out_sums), _ptr(out_bits), _stream(stream)))
    return out_sums, out_bits


def bnn_binarize_input(mode, x, offset=None, out=None, stream=None):
    """Input binarization (Sec. II-C): mode INPUT_THRESHOLD / INPUT_GRAY /
    INPUT_LBP on x [N,H,W,Cin] fp32 -> one code word per pixel [N,H,W,1]."""
    lib = load()
    _dev(x, torch.float32, "x")
    offset = _dev(offset, torch.float32, "offset")
    N, H, W, Cin = x.shape
    if out is None:
        out = _empty(x, (N, H, W, 1), torch.int32, stream)
    _check(lib.bnn_binarize_input(int(mode), _ptr(x), _ptr(offset), N, H, W, Cin, _ptr(out),
                                  _stream(stream)))
    return out


def bnn_bconv2d_input(desc: ConvDesc, mode, x, offset, w, thr=None, flip=None, want_sums=True,
                      want_bits=True, out_sums=None, out_bits=None, stream=None):
    """Binary conv over an fp32 image binarized on the fly by ``mode`` (Sec. II-C),
    each window packed into ceil(KH*KW*C / 32) words (Algorithm 1's patch
    packing).  desc.C is the binarized channel count.  Same outputs as
    bnn_binarize_input / bnn_pack_bits followed by bnn_bconv2d."""
    lib = load()
    Ho, Wo, Hp, Wp = _output_dims(desc)
    _dev(x, torch.float32, "x")
    offset = _dev(offset, torch.float32, "offset")
    _u32(w)
    thr = _dev(thr, torch.int32, "thr")
    flip = _dev(flip, torch.int32, "flip")
    if want_sums and out_sums is None:
        out_sums = _empty(x, (desc.N, Ho, Wo, desc.F), torch.int32, stream)
    if want_bits and out_bits is None:
        out_bits = _empty(x, (desc.N, Hp, Wp, words(desc.F)), torch.int32, stream)
    _check(lib.bnn_bconv2d_input(ctypes.byref(desc), int(mode), _ptr(x), _ptr(offset), _ptr(w),
                                 _ptr(thr), _ptr(flip), _ptr(out_sums), _ptr(out_bits),
                                 _stream(stream)))
    return out_sums, out_bits


def bnn_fconv_bconv2d(desc0: ConvDesc, desc1: ConvDesc, x, w0, thr0, flip0, w1, thr1,
                      flip1=None, out_bits=None, stream=None, w1prep=None):
    """The real-valued first layer and a binary 3x3 conv over its bits in one
    launch (the first two layers of Table I's BCNN): returns the second
    layer's packed bits [N, Hp, Wp, F1/32], the same as bnn_fconv2d_binw
    followed by bnn_bconv2d.  w1prep: bnn_prepare_weights of w1, or None."""
    lib = load()
    _, _, Hp, Wp = _output_dims(desc1)
    _dev(x, torch.float32, "x")
    _u32(w0)
    _u32(w1)
    thr0 = _dev(thr0, torch.int32, "thr0")
    thr1 = _dev(thr1, torch.int32, "thr1")
    flip0 = _dev(flip0, torch.int32, "flip0")
    flip1 = _dev(flip1, torch.int32, "flip1")
    if out_bits is None:
        out_bits = _empty(x, (desc1.N, Hp, Wp, words(desc1.F)), torch.int32, stream)
    _dev(w1prep, torch.uint8, "w1prep")
    _check(lib.bnn_fconv_bconv2d(ctypes.byref(desc0), ctypes.byref(desc1), _ptr(x), _ptr(w0),
                                 _ptr(thr0), _ptr(flip0), _ptr(w1), _ptr(w1prep), _ptr(thr1),
                                 _ptr(flip1), _ptr(out_bits), _stream(stream)))
    return out_bits


def bnn_input_bconv_bconv2d(desc0: ConvDesc, desc1: ConvDesc, mode, x, offset, w0, thr0, flip0,
                            w1, thr1, flip1=None, out_bits=None, stream=None, w1prep=None):
    """Input thresholding, a binary 3x3 conv and a binary 3x3 conv over its
    bits in one launch: returns the second conv's packed bits
    [N, Hp, Wp, F1/32], the same as bnn_bconv2d_input followed by
    bnn_bconv2d.  w1prep: bnn_prepare_weights of w1, or None."""
    lib = load()
    _, _, Hp, Wp = _output_dims(desc1)
    _dev(x, torch.float32, "x")
    offset = _dev(offset, torch.float32, "offset")
    _u32(w0)
    _u32(w1)
    thr0 = _dev(thr0, torch.int32, "thr0")
    thr1 = _dev(thr1, torch.int32, "thr1")
    flip0 = _dev(flip0, torch.int32, "flip0")
    flip1 = _dev(flip1, torch.int32, "flip1")
    if out_bits is None:
        out_bits = _empty(x, (desc1.N, Hp, Wp, words(desc1.F)), torch.int32, stream)
    _dev(w1prep, torch.uint8, "w1prep")
    _check(lib.bnn_input_bconv_bconv2d(ctypes.byref(desc0), ctypes.byref(desc1), int(mode),
                                       _ptr(x), _ptr(offset), _ptr(w0), _ptr(thr0), _ptr(flip0),
                                       _ptr(w1), _ptr(w1prep), _ptr(thr1), _ptr(flip1),
                                       _ptr(out_bits), _stream(stream)))
    return out_bits


def bnn_bconv_bconv2d(desc0: ConvDesc, desc1: ConvDesc, x, w0, thr0, flip0, w1, thr1,
                      flip1=None, out_bits=None, stream=None):
    """Two binary 3x3 convs in one launch, the first conv's bits kept on
    chip: returns the second conv's packed bits [N, Hp, Wp, F1/32], the same
    as bnn_bconv2d(desc0) followed by bnn_bconv2d(desc1)."""
    lib = load()
    _, _, Hp, Wp = _output_dims(desc1)
    _u32(x)
    _u32(w0)
    _u32(w1)
    thr0 = _dev(thr0, torch.int32, "thr0")
    thr1 = _dev(thr1, torch.int32, "thr1")
    flip0 = _dev(flip0, torch.int32, "flip0")
    flip1 = _dev(flip1, torch.int32, "flip1")
    if out_bits is None:
        out_bits = _empty(x, (desc1.N, Hp, Wp, words(desc1.F)), torch.int32, stream)
    _check(lib.bnn_bconv_bconv2d(ctypes.byref(desc0), ctypes.byref(desc1), _ptr(x), _ptr(w0),
                                 _ptr(thr0), _ptr(flip0), _ptr(w1), _ptr(thr1), _ptr(flip1),
                                 _ptr(out_bits), _stream(stream)))
    return out_bits


def bnn_bfc_pair(A, K0, w0, thr0, flip0, w1, N1, thr1=None, flip1=None, out=None,
                 stream=None):
    """Two binary FC layers in one launch: layer 0 (K0 -> N0 outputs, its
    threshold and flip) then layer 1 (N0 -> N1 <= 32).  With thr1 None the
    result is layer 1's int32 sums [M, N1]; otherwise its bits [M, 1].  The
    same as two bnn_bgemm calls."""
    lib = load()
    _u32(A)
    _u32(w0)
    _u32(w1)
    M, N0 = A.shape[0], w0.shape[0]
    thr0 = _dev(thr0, torch.int32, "thr0")
    flip0 = _dev(flip0, torch.int32, "flip0")
    thr1 = _dev(thr1, torch.int32, "thr1")
    flip1 = _dev(flip1, torch.int32, "flip1")
    if out is None:
        out = _empty(A, (M, N1) if thr1 is None else (M, 1), torch.int32, stream)
    _check(lib.bnn_bfc_pair(M, K0, N0, N1, _ptr(A), _ptr(w0), _ptr(thr0), _ptr(flip0), _ptr(w1),
                            _ptr(thr1), _ptr(flip1), _ptr(out) if thr1 is None else None,
                            None if thr1 is None else _ptr(out), _stream(stream)))
    return out


def bnn_bfc_tail(A, K0, w0, thr0, flip0, w1, N1, accum, thr1=None, flip1=None, out=None,
                 stream=None):
    """The FC tail kernel: the same two layers as bnn_bfc_pair, spread over
    layer 0's 32 x 32 output tiles, layer 1's partial sums added in `accum`
    (FORWARD_SYNC_BYTES, zero on entry and left zero: see accum_buffer)."""
    lib = load()
    _u32(A)
    _u32(w0)
    _u32(w1)
    M, N0 = A.shape[0], w0.shape[0]
    thr0 = _dev(thr0, torch.int32, "thr0")
    flip0 = _dev(flip0, torch.int32, "flip0")
    thr1 = _dev(thr1, torch.int32, "thr1")
    flip1 = _dev(flip1, torch.int32, "flip1")
    if out is None:
        out = _empty(A, (M, N1) if thr1 is None else (M, 1), torch.int32, stream)
    _check(lib.bnn_bfc_tail(M, K0, N0, N1, _ptr(A), _ptr(w0), _ptr(thr0), _ptr(flip0), _ptr(w1),
                            _ptr(thr1), _ptr(flip1), _ptr(out) if thr1 is None else None,
                            None if thr1 is None else _ptr(out), _ptr(accum), _stream(stream)))
    return out


def accum_buffer(device="cuda"):
    """A zeroed accumulator buffer for bnn_bfc_tail (FORWARD_SYNC_BYTES)."""
    return torch.zeros(FORWARD_SYNC_BYTES, dtype=torch.uint8, device=device)


def bnn_bgemm(A, B, K, thr=None, flip=None, want_sums=True, want_bits=True, out_sums=None,
              out_bits=None, stream=None):
    """Binary GEMM / FC (Sec. III-B): A [M,Kw], B [N,Kw] packed -> sums [M,N],
    bits [M,ceil(N/32)]."""
    lib = load()
    _u32(A)
    _u32(B)
    M, N = A.shape[0], B.shape[0]
    thr = _dev(thr, torch.int32, "thr")
    flip = _dev(flip, torch.int32, "flip")
    if want_sums and out_sums is None:
        out_sums = _empty(A, (M, N), torch.int32, stream)
    if want_bits and out_bits is None:
        out_bits = _empty(A, (M, words(N)), torch.int32, stream)
    _check(lib.bnn_bgemm(M, N, K, _ptr(A), _ptr(B), _ptr(thr), _ptr(flip), _ptr(out_sums),
                         _ptr(out_bits), _stream(stream)))
    return out_sums, out_bits


# ---------------------------------------------- mixtures of binary experts ---
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.int32: 3}
_SCORES = {"softmax": 0, "sigmoid": 1}


def _real(dtype, name):
    code = _DTYPES.get(dtype)
    if code is None or code == 3:
        raise TypeError("%s must be float32, float16 or bfloat16" % name)
    return code


def _shaped(t, shape, name):
    if t is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, shape, tuple(t.shape)))
    return t


def _output(t, like, shape, dtype, name, stream):
    """A new tensor on like's device, or the caller's, looked at."""
    if t is None:
        return _empty(like, shape, dtype, stream)
    return _shaped(_dev(t, dtype, name), shape, name)


def _rows(t, name):
    """A 2-d tensor whose rows are contiguous and do not overlap: their distance
    in elements."""
    if t.dim() != 2 or not t.is_cuda or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be a 2-d CUDA(HIP) tensor with contiguous rows" % name)
    if t.shape[0] < 2:
        return t.shape[1]
    if t.stride(0) < t.shape[1]:
        raise ValueError("the rows of %s overlap (%d elements long, %d apart): call contiguous()"
                         % (name, t.shape[1], t.stride(0)))
    return t.stride(0)


# (The sizes of workspaces are functions of the call's sizes alone: asked for
# once for each, 0.6 us a call.)
def _workspace(ws, need, like, stream):
    """The caller's workspace, or a new one of `need` bytes beside like, and its
    size."""
    if ws is None:
        return (_scratch(like, need, torch.uint8, stream) if need else None), need
    return ws, _dev(ws, torch.uint8, "workspace").numel()


def bnn_route(logits, top_k, bias=None, score="softmax", groups=1, top_groups=None, group_top=1,
              renormalize=True, scale=1.0, logit_scale=1.0, ids=None, weights=None, stream=None):
    """Routing: logits [T, E] (float32, float16, bfloat16 or int32; rows may be
    strided) -> (ids [T, top_k] int32, weights [T, top_k] float32).  The
    experts of the largest p + bias (p: softmax or sigmoid of logit_scale *
    logits), with groups > 1 out of the top_groups groups of the largest
    scores; weights are scale * p, with renormalize over the chosen experts'
    sum.  Experts out of reach (logit -inf) are never chosen: id -1."""
    lib = load()
    dtype = _DTYPES.get(logits.dtype)
    if dtype is None:
        raise TypeError("logits must be float32, float16, bfloat16 or int32")
    stride = _rows(logits, "logits")
    T, E = logits.shape
    bias = _shaped(_dev(bias, torch.float32, "bias"), (E,), "bias")
    ids = _output(ids, logits, (T, top_k), torch.int32, "ids", stream)
    weights = _output(weights, logits, (T, top_k), torch.float32, "weights", stream)
    if score not in _SCORES:
        raise ValueError("score must be one of %s" % sorted(_SCORES))
    d = RouteDesc(E, top_k, groups, groups if top_groups is None else top_groups, group_top,
                  _SCORES[score], bool(renormalize), dtype, scale, logit_scale)
    _check(lib.bnn_route(ctypes.byref(d), T, _ptr(logits), stride, _ptr(bias), _ptr(ids),
                         _ptr(weights), _stream(stream)))
    return ids, weights


def bnn_group_rows_workspace_size(M, G) -> int:
    out = ctypes.c_size_t()
    _check(load().bnn_group_rows_workspace_size(M, G, ctypes.byref(out)))
    return out.value


_group_rows_bytes = functools.lru_cache(maxsize=1024)(bnn_group_rows_workspace_size)


def bnn_group_rows(ids, G, offsets=None, order=None, workspace=None, stream=None):
    """Rows in the order of their group: ids (any shape, int32) -> (offsets
    [G + 1], order [ids.numel()]) int32; rows whose id is not in [0, G) come
    last."""
    lib = load()
    _dev(ids, torch.int32, "ids")
    M = ids.numel()
    offsets = _output(offsets, ids, (G + 1,), torch.int32, "offsets", stream)
    order = _output(order, ids, (M,), torch.int32, "order", stream)
    workspace, n = _workspace(workspace, _group_rows_bytes(M, G), ids, stream)
    _check(lib.bnn_group_rows(M, G, _ptr(ids), _ptr(offsets), _ptr(order), _ptr(workspace), n,
                              _stream(stream)))
    return offsets, order


def _experts_desc(x, K, w, M, top_k, offsets, order):
    """The description of M = T * top_k pairs over x [T, Kw] or [M, Kw]."""
    _u32(x)
    _u32(w)
    E, N, kw = w.shape
    T = M // top_k
    if x.dim() != 2 or x.shape[1] != kw or kw != words(K) or x.shape[0] not in (T, M):
        raise ValueError("x must be [%d or %d, %d] packed words of %d bits" % (T, M, words(K), K))
    _shaped(_dev(offsets, torch.int32, "offsets"), (E + 1,), "offsets")
    _shaped(_dev(order, torch.int32, "order"), (M,), "order")
    return ExpertsDesc(T, top_k, E, N, K, int(top_k > 1 and x.shape[0] == T))


def bnn_experts_fc(x, K, w, offsets, order, thr, flip=None, out_bits=None, stream=None):
    """Binary FC layers of experts, to bits: x [T, Kw] (a row's experts read
    the same bits) or [M, Kw], M = order.numel() (row, expert) pairs; w
    [E, N, Kw], thr [E, N], flip [E, ceil(N/32)]; offsets and order of
    bnn_group_rows -> bits [M, ceil(N/32)] (0 for a pair without an expert)."""
    lib = load()
    M, rows = order.numel(), x.shape[0]
    if M and (not rows or M % rows):
        raise ValueError("%d pairs do not go evenly over %d rows of x" % (M, rows))
    d = _experts_desc(x, K, w, M, M // rows if M else 1, offsets, order)
    nw = words(d.N)
    _shaped(_dev(thr, torch.int32, "thr"), (d.E, d.N), "thr")
    _shaped(_dev(flip, torch.int32, "flip"), (d.E, nw), "flip")
    out_bits = _output(out_bits, x, (M, nw), torch.int32, "out_bits", stream)
    _check(lib.bnn_experts_fc(ctypes.byref(d), _ptr(x), _ptr(w), _ptr(offsets), _ptr(order),
                              _ptr(thr), _ptr(flip), _ptr(out_bits), _stream(stream)))
    return out_bits


def bnn_experts_sum_workspace_size(desc: ExpertsDesc) -> int:
    out = ctypes.c_size_t()
    _check(load().bnn_experts_sum_workspace_size(ctypes.byref(desc), ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=1024)
def _experts_sum_bytes(*sizes):
    return bnn_experts_sum_workspace_size(ExpertsDesc(*sizes))


def bnn_experts_sum(x, K, w, ids, weights, offsets, order, alpha=None, dtype=torch.float32,
                    out=None, workspace=None, stream=None):
    """Binary FC layers of experts, weighted and added up per row: ids and
    weights [T, top_k] (of bnn_route), x [T * top_k, Kw] or [T, Kw], w
    [E, N, Kw], alpha [E, N] float32; offsets and order of bnn_group_rows(ids)
    -> y [T, N] of dtype, y[t] = sum_j weights[t, j] * alpha[e] * S[t, j]."""
    lib = load()
    _dev(ids, torch.int32, "ids")
    T, top_k = ids.shape
    _shaped(_dev(weights, torch.float32, "weights"), (T, top_k), "weights")
    d = _experts_desc(x, K, w, T * top_k, top_k, offsets, order)
    _shaped(_dev(alpha, torch.float32, "alpha"), (d.E, d.N), "alpha")
    dtype = dtype if out is None else out.dtype
    code = _real(dtype, "out")
    out = _output(out, x, (T, d.N), dtype, "out", stream)
    workspace, n = _workspace(
        workspace, _experts_sum_bytes(T, top_k, d.E, d.N, d.K, d.share), x, stream)
    _check(lib.bnn_experts_sum(ctypes.byref(d), _ptr(x), _ptr(w), _ptr(ids), _ptr(weights),
                               _ptr(offsets), _ptr(order), _ptr(alpha), code, _ptr(out),
                               _ptr(workspace), n, _stream(stream)))
    return out


def bnn_bgemm_lora_workspace_size(desc: LoraDesc) -> int:
    out = ctypes.c_size_t()
    _check(load().bnn_bgemm_lora_workspace_size(ctypes.byref(desc), ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=1024)
def _lora_bytes(*sizes):
    return bnn_bgemm_lora_workspace_size(LoraDesc(*sizes))


def bnn_bgemm_lora(x, w, ids, a, b, scale=None, alpha=None, offset=None, order=None, dtype=None,
                   out=None, workspace=None, stream=None):
    """A binary FC layer with a low-rank adapter per row: x [M, K] (float32,
    float16 or bfloat16; rows may be strided), w [N, Kw] packed, ids [M] the
    rows' adapters (-1: none), a [L, rank, K] and b [L, N, rank] of x's type,
    scale [L], alpha [N], offset [K] float32 -> y [M, N] of dtype (x's),
    y = alpha * (sign(x + offset) . w) + scale[l] * (x a[l]^T) b[l]^T.
    order: bnn_group_rows(ids, L)[1], or None."""
    lib = load()
    kind = x.dtype
    code = _real(kind, "x")
    stride = _rows(x, "x")
    M, K = x.shape
    _u32(w)
    N = w.shape[0]
    _shaped(w, (N, words(K)), "w")
    if _dev(a, kind, "a").dim() != 3:
        raise ValueError("a must have shape [adapters, rank, %d], got %s" % (K, tuple(a.shape)))
    L, rank = a.shape[0], a.shape[1]
    _shaped(a, (L, rank, K), "a")
    _shaped(_dev(b, kind, "b"), (L, N, rank), "b")
    _shaped(_dev(ids, torch.int32, "ids"), (M,), "ids")
    _shaped(_dev(order, torch.int32, "order"), (M,), "order")
    _shaped(_dev(scale, torch.float32, "scale"), (L,), "scale")
    _shaped(_dev(alpha, torch.float32, "alpha"), (N,), "alpha")
    _shaped(_dev(offset, torch.float32, "offset"), (K,), "offset")
    dtype = out.dtype if out is not None else kind if dtype is None else dtype
    out_code = _real(dtype, "out")
    out = _output(out, x, (M, N), dtype, "out", stream)
    d = LoraDesc(M, N, K, L, rank, code, out_code)
    workspace, n = _workspace(workspace, _lora_bytes(M, N, K, L, rank, code, out_code), x,
                              stream)
    _check(lib.bnn_bgemm_lora(ctypes.byref(d), _ptr(x), stride, _ptr(offset), _ptr(w),
                              _ptr(alpha), _ptr(ids), _ptr(a), _ptr(b), _ptr(scale), _ptr(order),
                              _ptr(out), _ptr(workspace), n, _stream(stream)))
    return out


class Network:
    """A layer chain for bnn_forward.  ``layers`` holds dicts with the C
    struct's fields and device tensors (w, thr, flip, offset); the tensors are
    kept alive by this object."""

    def __init__(self, layers, H, W, C):
        self.H, self.W, self.C = H, W, C
        self._tensors = layers
        arr = (Layer * len(layers))()
        for i, d in enumerate(layers):
            L = arr[i]
            L.kind = d["kind"]
            for f in ("C", "F", "KH", "KW", "stride", "pad", "pool", "K", "N"):
                setattr(L, f, int(d.get(f, 0)))
            for f in ("w", "thr", "flip", "offset", "wprep"):
                t = d.get(f)
                setattr(L, f, None if t is None else t.data_ptr())
        self.layers = arr
        self.n = len(layers)

    def workspace_size(self, batch: int) -> int:
        lib = load()
        out = ctypes.c_size_t()
        _check(lib.bnn_forward_workspace_size(self.layers, self.n, batch, self.H, self.W,
                                              self.C, ctypes.byref(out)))
        return out.value

    def alloc_workspace(self, batch: int, device="cuda"):
        """A bnn_forward workspace for `batch` images, its accumulator bytes zeroed."""
        ws = torch.empty(self.workspace_size(batch), dtype=torch.uint8, device=device)
        ws[:FORWARD_SYNC_BYTES].zero_()
        return ws


def bnn_forward(net: Network, x, workspace=None, logits=None, stream=None):
    """Run the chain on x [batch, H, W, C] fp32; returns int32 logits."""
    lib = load()
    _dev(x, torch.float32, "x")
    batch = x.shape[0]
    if workspace is None:
        # (zeroed on the stream that reads it)
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            workspace = net.alloc_workspace(batch, x.device)
    n_out = net.layers[net.n - 1].N
    if logits is None:
        logits = _empty(x, (batch, n_out), torch.int32, stream)
    _check(lib.bnn_forward(net.layers, net.n, batch, net.H, net.W, net.C, _ptr(x),
                           _ptr(workspace), workspace.numel(), _ptr(logits),
                           _stream(stream)))
    return logits


def bnn_forward_noalloc(net: Network, x, logits=None, stream=None):
    """bnn_forward with the intermediate bits in the library's per-GPU scratch
    array instead of a workspace (for callers that cannot allocate); returns
    int32 logits."""
    lib = load()
    _dev(x, torch.float32, "x")
    batch = x.shape[0]
    n_out = net.layers[net.n - 1].N
    if logits is None:
        logits = _empty(x, (batch, n_out), torch.int32, stream)
    _dev(logits, torch.int32, "logits")
    _check(lib.bnn_forward_noalloc(net.layers, net.n, batch, net.H, net.W, net.C, _ptr(x),
                                   _ptr(logits), _stream(stream)))
    return logits


# Short aliases.
pack_bits = bnn_pack_bits
bconv2d = bnn_bconv2d
fconv2d_binw = bnn_fconv2d_binw
bconv2d_input = bnn_bconv2d_input
fconv_bconv2d = bnn_fconv_bconv2d
binarize_input = bnn_binarize_input
bgemm = bnn_bgemm
route = bnn_route
group_rows = bnn_group_rows
experts_fc = bnn_experts_fc
experts_sum = bnn_experts_sum
bgemm_lora = bnn_bgemm_lora
forward = bnn_forward
