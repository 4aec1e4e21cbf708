"""What the compiler says of the 4-bit append's kernels: arrays of values stay in registers."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_append_keeps_its_values_in_registers(tmp_path):
    src = tmp_path / "append.cu"
    src.write_text('#include "subgen_paged.cuh"\n' + "".join(
        "template __global__ void sgk::norm_rope_kernel<%s, %d, 2, %d>(sgk::NormRope, sgk::PagedView);\n" % (t, d, u)
        for t in ("float", "__nv_bfloat16") for d in (64, 128) for u in (1, 4)))
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    said = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas", "-v", "-cubin", "-o", str(tmp_path / "append.cubin"),
                           "-I" + os.path.join(ROOT, "paper_2402_06082_b200", "csrc"), str(src)], capture_output=True, text=True, check=True).stderr
    frames = [[int(x) for x in m] for m in re.findall(r"(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", said)]
    assert len(frames) == 8, said
    for frame, stored, _ in frames:                          # what is on the stack is a few spilled words, no array
        assert frame <= stored <= 48, said
