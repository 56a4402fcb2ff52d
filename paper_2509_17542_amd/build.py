"""Build step of the HIP library: compiles csrc/ into libkvx.so for gfx950.

    python -m paper_2509_17542_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libkvx.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# -packed-fp32-ops: no v_pk_{add,mul,fma}_f32 are generated.
# -ffp-contract=off: no fused multiply-adds beyond the explicit ones.
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-ffp-contract=off", "-I", INCLUDE, "-I", CSRC]
DEVICE = ["-x", "hip", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
          "-packed-fp32-ops"]
SOURCES = [("kvx_kernels.hip", True), ("kvx_plan.cpp", False), ("kvx_pipe.cpp", False),
           ("kvx_pd.cpp", False), ("kvx_ops.cpp", False), ("kvx_slots.hip", True),
           ("kvx_attend.hip", True), ("kvx_attend_few.hip", True),
           ("kvx_attend_rows_16.hip", True), ("kvx_attend_rows_e4m3.hip", True),
           ("kvx_attend_rows_e5m2.hip", True), ("kvx_weigh.hip", True)]


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs, todo = [], []
    for name, device in SOURCES:
        obj = os.path.join(BUILD, name + ".o")
        cmd = [HIPCC] + COMMON + (DEVICE if device else ["-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include"]) + \
            ["-c", os.path.join(CSRC, name), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        todo.append(cmd)
        objs.append(obj)
    with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        list(pool.map(lambda c: subprocess.run(c, check=True), todo))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "--offload-arch=gfx950", "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
