"""Compile the CUDA library in-tree for sm_100a with nvcc (no JIT cache, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsubgen.so")
SOURCES = ["subgen.cu", "subgen_paged.cu"]
HEADERS = ["subgen_device.cuh", "subgen_kernels.cuh", "subgen_query_mma.cuh", "subgen_insert_mma.cuh", "subgen_step_fused.cuh", "subgen_prefill.cuh", "subgen_score_tc.cuh", "subgen_prefill_persist.cuh", "subgen_exact_mma.cuh", "subgen_kcenter.cuh", "subgen_paged.cuh", "subgen_paged_simt.cuh", "subgen_paged_tc.cuh", os.path.join("..", "..", "include", "subgen.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", str(len(SOURCES)),
           "-shared", "-Xcompiler", "-fPIC", "-o", LIB + ".tmp"] + [os.path.join(CSRC, f) for f in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
