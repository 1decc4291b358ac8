"""How the log probabilities' rows are spread (csrc/logprobs_plans.hpp, host
code): the plans fit their sizes and the kernels' limits, and the GPU tests reach
every form (CPU only)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import test_gpu_logprobs_forms as forms
import tile_plans

SHIM = r"""
#include "logprobs_plans.hpp"
extern "C" void plan(int64_t T, int V, int64_t* out) {
  const bnn::LogprobsPlan p = bnn::logprobs_plan(T, V);
  out[0] = p.waves; out[1] = p.splits; out[2] = p.length; out[3] = bnn::logprobs_parts(T, V);
}
"""
STEP = 1024


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory(prefix="logprobs_plans_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", tile_plans.CSRC, src,
                        "-o", so], check=True)
        return ctypes.CDLL(so)


def _plan(T, V):
    out = (ctypes.c_int64 * 4)()
    lib().plan(ctypes.c_int64(T), V, out)
    return tuple(out)


def _form(T, V):
    waves, splits, length, _ = _plan(T, V)
    last = V - (splits - 1) * length  # values of the last part
    return (waves, "row" if splits == 1 else "parts" if splits <= 64 else "many parts",
            "whole" if last % (waves * STEP) == 0 else "groups" if last % 8 == 0 else "odd")


def test_plans_fit():
    for V in (1, 7, 1023, 1024, 1025, 4096, 4097, 8192, 8193, 12289, 16384, 65536, 100003, 300001, 1 << 24):
        parts = 0
        for T in (1, 2, 3, 15, 16, 50, 159, 160, 511, 512, 2047, 2048, 5000, (1 << 24) - 1):
            waves, splits, length, room = _plan(T, V)
            assert waves in (1, 4, 16) and length % STEP == 0
            assert splits * length >= V and (splits == 1 or T < 160 and waves == 4)
            assert splits == 1 or (splits * T <= room and splits * T < 1 << 31)
            assert room >= parts  # (of any fewer rows)
            parts = room
            rows = -(-T * splits // (4 if waves == 1 else 1))  # workgroups
            assert rows * (1024 if waves == 16 else 256) < 1 << 32
            assert waves != 16 or T < 512


def test_every_form_is_reached():
    reached = {_form(T, V) for T, V in forms.SIZES}
    assert {f[:2] for f in reached} == {(1, "row"), (4, "row"), (16, "row"), (4, "parts"), (4, "many parts")}
    assert {f for f in reached if f[0] == 16} == {(16, "row", end) for end in ("whole", "groups", "odd")}
    assert any(_plan(T, V)[1] > 64 for T, V in forms.SIZES) and any(_plan(T, V)[2] % 4096 for T, V in forms.SIZES)


def test_measured_choices():
    assert _plan(16384, 1000)[:2] == (1, 1) and _plan(4096, 131072)[:2] == (4, 1)
    assert _plan(301, 50021)[:2] == (16, 1) and _plan(1, 65536)[:3] == (4, 16, 4096)
    assert _plan(1000, 4096)[0] == 4 and _plan(4000, 4096)[0] == 1
    assert _plan(1, 8193)[1:3] == (3, 3072) and _plan(64, 8000)[1] == 1
