"""Compile the CUDA library in-tree for sm_100a with nvcc, and the Python calls module with g++ (no JIT cache, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsubgen.so")
CALLS = os.path.join(HERE, "_calls.so")
CALLS_SOURCES = ["calls.cpp", os.path.join("..", "..", "include", "subgen.h")]
SOURCES = ["subgen.cu", "subgen_paged.cu", "subgen_paged4.cu"]
HEADERS = ["subgen_device.cuh", "subgen_kernels.cuh", "subgen_query_mma.cuh", "subgen_insert_mma.cuh", "subgen_step_fused.cuh", "subgen_prefill.cuh", "subgen_score_tc.cuh", "subgen_prefill_persist.cuh", "subgen_exact_mma.cuh", "subgen_kcenter.cuh", "subgen_paged.cuh", "subgen_paged_simt.cuh", "subgen_paged_tc.cuh", "subgen_paged_host.cuh", "subgen_codes4.cuh", "subgen_paged4.cuh", "subgen_paged4_few.cuh", os.path.join("..", "..", "include", "subgen.h")]


def _stale(out: str, sources) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in sources)


def built_for() -> str:
    """What the calls module depends on besides its sources; compiled into it."""
    import torch
    return "torch %s, python %d.%d" % (torch.__version__, *sys.version_info[:2])


def _calls_stale() -> bool:
    if _stale(CALLS, CALLS_SOURCES):
        return True
    with open(CALLS, "rb") as f:
        return ("built for " + built_for()).encode() + b"\0" not in f.read()


def _calls_command(out: str):
    """calls.cpp against the headers and libraries of the torch that runs this."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), sysconfig.get_paths()["include"]]
    lib = os.path.join(root, "lib")
    return (["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
             '-DSUBGEN_BUILT_FOR="built for %s"' % built_for()]
            + ["-I" + d for d in inc] + ["-o", out, os.path.join(CSRC, "calls.cpp"), "-L" + lib]
            + ["-l" + x for x in ("torch_python", "torch", "torch_cpu", "c10", "c10_cuda")] + ["-Wl,-rpath," + lib])


def build(force: bool = False, verbose: bool = False) -> str:
    jobs = []
    if force or _stale(LIB, SOURCES + HEADERS):
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", str(len(SOURCES)),
               "-shared", "-Xcompiler", "-fPIC", "-o", LIB + ".tmp"] + [os.path.join(CSRC, f) for f in SOURCES]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        jobs.append((LIB, cmd, subprocess.Popen(cmd)))
    if force or _calls_stale():
        cmd = _calls_command(CALLS + ".tmp")
        jobs.append((CALLS, cmd, subprocess.Popen(cmd)))
    codes = [p.wait() for _, _, p in jobs]
    for (out, cmd, _), rc in zip(jobs, codes):
        if rc:
            raise subprocess.CalledProcessError(rc, cmd)
        os.replace(out + ".tmp", out)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
