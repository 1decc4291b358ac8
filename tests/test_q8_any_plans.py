"""The tiles of the 8-bit product of rows that lie anywhere (csrc/q8_plans.hpp,
host code): the GPU tests reach both with every kind of K (CPU only)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import test_gpu_q8gemm_any as gpu
import tile_plans

SHIM = r"""
#include "q8_plans.hpp"
extern "C" int form(int64_t M, int64_t N, int64_t K, int on16) { return bnn::q8_form(M, N, K, on16); }
extern "C" int on16(int64_t at, int64_t stride, int64_t rows) { return bnn::q8_on16(at, stride, rows); }
extern "C" int tile(int64_t M, int64_t N) { return bnn::q8_any_tile(M, N); }
"""


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory(prefix="q8_any_plans_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", tile_plans.CSRC, src,
                        "-o", so], check=True)
        return ctypes.CDLL(so)


def _tile(M, N):
    return lib().tile(ctypes.c_int64(M), ctypes.c_int64(N))


def _any(M, N, K):
    return lib().form(ctypes.c_int64(M), ctypes.c_int64(N), ctypes.c_int64(K), ctypes.c_int(0)) == 0


def test_both_tiles_are_reached():
    assert {_tile(M, N) for M, N in gpu.LARGE} == {128} and {_tile(M, N) for M, N in gpu.SMALL} == {64}
    for sizes, tile in ((gpu.LARGE, 128), (gpu.SMALL, 64)):
        for M, N in sizes:
            for K in gpu.KS:
                assert _any(M, N, K + 8192 if M <= 16 and K >= 16 else K)
    assert any(K < 16 for K in gpu.KS) and any(16 <= K < 128 for K in gpu.KS)
    assert any(K % 128 == 0 for K in gpu.KS) and any(K > 128 and K % 16 for K in gpu.KS)
    assert _any(2050, 2060, 1024) and _tile(2050, 2060) == 128


def test_launches_fit():
    """Work-items of a launch stay below 2^32 at the most outputs a call may have."""
    for M in (1, 16, 65, 4097, 1 << 15, 1 << 20, (1 << 24) - 1):
        N = min(1 << 20, (1 << 35) // M)
        tile = _tile(M, N)
        assert -(-M // tile) * -(-N // tile) * 256 < 1 << 32


def test_one_row_has_no_distance():
    on16 = lambda *a: bool(lib().on16(*map(ctypes.c_int64, a)))  # noqa: E731
    assert on16(0x1000, 14335, 1) and on16(0x1000, 14336, 2) and on16(0x10, 16, 9)
    assert not on16(0x1000, 14335, 2) and not on16(0x1008, 14336, 2) and not on16(0x1001, 14335, 1)
