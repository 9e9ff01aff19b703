"""Builds libmoe_gfx950.so (HIP kernels + C ABI) in-tree with hipcc.  gfx950 only."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmoe_gfx950.so")
SOURCES = ["moe_api.hip", "moe_route.hip", "moe_permute.hip", "moe_pack.hip", "moe_gemm.hip", "moe_gemm_swiglu.hip",
           "moe_gemm_plain.hip", "moe_gemm_pairsum.hip", "moe_gemm_partial.hip", "moe_gemm_swiglu_stream.hip",
           "moe_gemm_plain_stream.hip", "moe_gemm_partial_stream.hip", "moe_place.hip",
           "moe_ops_api.hip", "moe_grouped.hip", "moe_grouped_row_major.hip", "moe_grouped_transposed.hip", "moe_grouped_mx.hip",
           "moe_grouped_weights.hip", "moe_mxfp4.hip", "moe_swiglu.hip", "moe_grad_norm.hip"]
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


def _hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def build(verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    hipcc = _hipcc()
    if os.path.exists(LIB):
        os.remove(LIB)          # never leave a stale library behind a failed build

    def compile_one(src):
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    r = subprocess.run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
