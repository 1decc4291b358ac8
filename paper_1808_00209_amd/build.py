"""Build libbnn.so (HIP kernels + C ABI) for gfx950 with hipcc.

Usage: ``python -m paper_1808_00209_amd.build`` (always recompiles).
Every source is compiled with the packed-fp32 instructions switched off, with
fp32 denormals kept (the sign test ``x > 0`` must see them) and with MFMA
accumulators in VGPRs.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libbnn.so")
BUILD_DIR = os.path.join(PKG, "_build")

SOURCES = ["pack.hip", "bconv_valu.hip", "bconv_mfma.hip", "bconv_tile.hip", "bconv_1x1.hip",
           "bconv_patch.hip", "fconv.hip", "fconv_bconv.hip", "bconv_bconv.hip", "bfc_chain.hip",
           "bfc_pair.hip", "bfc_gemm.hip", "bfc_tile.hip", "route.hip", "group_rows.hip",
           "experts.hip", "experts_tile.hip", "experts_skinny.hip",
           "experts_combine.hip", "experts_sum_rows.hip",
           "lora.hip", "lora_tile.hip", "lora_skinny.hip", "rmsnorm.hip", "q8gemm.hip",
           "q8gemm_skinny.hip", "q8gemm_tile.hip", "logprobs.hip",
           "api.cpp", "experts_api.cpp", "quant_api.cpp"]
ARCH = os.environ.get("BNN_OFFLOAD_ARCH", "gfx950")

COMMON = [
    "-O3", "-fPIC", "-std=c++17", "--offload-arch=" + ARCH,
    "-I", INCLUDE, "-I", CSRC,
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fno-gpu-flush-denormals-to-zero", "-ffp-contract=off",
    # MFMA accumulators stay in VGPRs (the AGPR form made the compiler copy
    # every accumulator out and back around each MFMA of the conv loop).
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _compile(src: str, extra=()) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [hipcc(), *COMMON, *extra, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), r.stderr))
    # (hipcc's host pass does not know the feature that its device pass takes)
    told = [line for line in r.stderr.splitlines() if "packed-fp32-ops" not in line]
    if told:
        print("%s:\n%s" % (src, "\n".join(told)), file=sys.stderr)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc(), "-shared", "-fPIC", "--offload-arch=" + ARCH, *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
