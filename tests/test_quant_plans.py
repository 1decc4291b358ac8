"""The choice of kernels of the 8-bit matrix product (csrc/q8_plans.hpp, host
code): which form each size of the GPU tests takes, so that together they reach
every one (CPU only)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import test_gpu_q8gemm as q8
import tile_plans

SHIM = r"""
#include "q8_plans.hpp"
extern "C" int form(int64_t M, int64_t N, int64_t K, int on16) { return bnn::q8_form(M, N, K, on16); }
"""
ANY, SKINNY, TILE64, TILE128, PAIR128, TILE256 = range(6)


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory(prefix="q8_plans_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", tile_plans.CSRC, src,
                        "-o", so], check=True)
        return ctypes.CDLL(so)


def _form(M, N, K, on16=True):
    return lib().form(ctypes.c_int64(M), ctypes.c_int64(N), ctypes.c_int64(K), ctypes.c_int(on16))


def test_every_form_is_reached():
    """Each tile with K shorter than a stage of 128, of whole stages, and with a
    short last stage of whole 16-byte chunks and of a part of one."""
    reached = {(_form(M, N, K), "short" if K < 128 else "whole" if K % 128 == 0 else
                "chunks" if K % 16 == 0 else "part") for M, N, K in q8.SIZES}
    for form in (TILE64, TILE128, PAIR128, TILE256):
        assert {kind for f, kind in reached if f == form} == {"short", "whole", "chunks", "part"}, form
    assert {f for f, _ in reached} == set(range(6))
    assert {_form(M, 200, K, False) for M in (1, 9, 40, 130, 700) for K in (15, 16, 17, 1001)} == {ANY, SKINNY}


def test_forms_fit_their_sizes():
    for M in (1, 16, 17, 32, 33, 64, 65, 500, 5000, (1 << 24) - 1):
        for N in (1, 63, 2048, 1 << 20):
            for K in (1, 15, 16, 4096, 4097, 8192, 8193, 131071):
                for on16 in (False, True):
                    f = _form(M, N, K, on16)
                    if f == SKINNY:  # x in registers: 16 steps of 64 per wave
                        assert 16 <= K <= 8192 and M <= 16
                    elif f != ANY:
                        assert K >= 16 and on16
                    else:
                        assert K < 16 or not on16


def test_measured_choices():
    assert _form(256, 4096, 4096) == TILE64 and _form(777, 2050, 1100) == TILE64
    assert _form(1024, 4096, 4096) == TILE128 and _form(2048, 4096, 4096) == PAIR128
    assert _form(4096, 4096, 4096) == TILE256 and _form(8192, 16384, 4096) == TILE256
    assert _form(16, 65536, 4096) == SKINNY and _form(17, 65536, 4096) != SKINNY
