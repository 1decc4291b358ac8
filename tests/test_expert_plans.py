"""The choice of kernels of the mixture-of-experts calls (csrc/expert_plans.hpp,
host code): which form each case of the GPU tests reaches, so that together
they reach every one (CPU only)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import test_gpu_experts as experts
import test_gpu_lora as lora
import tile_plans

SHIM = r"""
#include "expert_plans.hpp"
using namespace bnn;
static void put(const TileShape& s, int* o) { o[0] = s.wfl; o[1] = s.pt; }
extern "C" {
int sum_by_rows(int64_t M, int64_t N, int64_t K) { return experts_sum_by_rows(M, N, K); }
int skinny(int64_t M, int64_t E, int64_t N) { return experts_skinny(M, E, N); }
void experts_tile(int64_t M, int64_t E, int64_t N, int64_t K, int* o) {
  put(experts_shape(M, E, N, (K + 255) / 256), o);
}
int combine(int64_t T, int64_t E, int64_t N) { return combine_rows(T, E, N); }
int down_rows(int64_t M, int64_t rank) { return lora_down_by_rows(M, rank); }
int down_slices(int64_t M, int64_t K, int64_t rank) { return lora_down_slices(M, K, rank); }
int up_skinny(int64_t M, int64_t N) { return lora_up_skinny(M, N); }
void lora_tile(int64_t M, int64_t N, int64_t K, int* o) { put(lora_shape(M, N, (K + 255) / 256), o); }
}
"""


@functools.lru_cache(maxsize=None)
def lib():
    with tempfile.TemporaryDirectory(prefix="expert_plans_") as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", tile_plans.CSRC, src,
                        "-o", so], check=True)
        return ctypes.CDLL(so)


def _call(name, *args):
    return getattr(lib(), name)(*[ctypes.c_int64(a) for a in args])


def _shape(name, *args):
    o = (ctypes.c_int * 2)()
    getattr(lib(), name)(*[ctypes.c_int64(a) for a in args], o)
    return tuple(o)


SHAPES = {(0, 1), (1, 1), (1, 2), (2, 1), (2, 2), (2, 4)}  # waves along the outputs, row tiles


def test_shapes_stay_within_the_staged_rows():
    for N in (1, 64, 65, 700, 4096):
        for M in (1, 40, 1000, 100000):
            for K in (1, 1024, 65535):
                for s in (_shape("lora_tile", M, N, K), _shape("experts_tile", M, 8, N, K)):
                    assert s in SHAPES


def test_the_experts_cases_reach_every_form():
    seen, waves = set(), set()
    def form(T, k, E, K, N, _):
        return "skinny" if _call("skinny", T * k, E, N) else _shape("experts_tile", T * k, E, N, K)

    for case in experts.CASES + experts.LARGE:
        T, k, E, K, N, _ = case
        if not _call("sum_by_rows", T * k, N, K):
            seen.add(("sum", form(*case)))
            seen.add("staged" if _call("combine", T, E, N) else "direct")
        else:
            seen.add("rows")
    for case in experts.CASES + experts.LARGE[:8] + experts.TILES:
        seen.add(("bits", form(*case)))
        if form(*case) == "skinny":
            chunks = (case[3] + 255) // 256
            waves.add(8 if chunks > 4 else 4 if chunks > 2 else 2)
    assert {"rows", "staged", "direct", ("sum", "skinny"), ("bits", "skinny")} <= seen
    assert waves == {2, 4, 8}
    for kind in ("sum", "bits"):
        reached = {s[1] for s in seen if isinstance(s, tuple) and s[0] == kind} - {"skinny"}
        assert reached == SHAPES, kind


def test_the_adapter_cases_reach_every_form():
    down, up = set(), set()
    for M, K, N, _, rank, kind, _ in lora.CASES:
        if _call("down_rows", M, rank):
            down.add("rows")
            assert _call("down_slices", M, K, rank) == 1
        else:
            n = _call("down_slices", M, K, rank)
            down.add((1 if rank <= 16 else 2 if rank <= 32 else 4, n > 1))
        up.add("skinny" if _call("up_skinny", M, N) else _shape("lora_tile", M, N, K))
    assert "rows" in down
    assert {d[0] for d in down if d != "rows"} == {1, 2, 4}  # 16-rank tiles per block
    assert {d[1] for d in down if d != "rows"} == {False, True}  # k in slices
    assert "skinny" in up
    assert up - {"skinny"} == SHAPES
