"""The C++ calls module is bound by the paged functions alone: SubGen and the exact cache do without it."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT = """
import sys
sys.modules["paper_2402_06082_b200._calls"] = None    # an import of it fails
import torch
from paper_2402_06082_b200 import binding
L = binding.load()
assert L.subgen_workspace_bytes(binding.SubgenConfig(2, 4, 4, 128, 0.5, 8, 64, 16, 0, binding.DTYPE_BF16, 128, 0, None, 0, None)) > 0
binding.Rope(64, device="cpu")
try:
    binding.qk_norm_rope(torch.zeros(1, 1, 64), None)
except RuntimeError as e:
    assert "_calls.so" in str(e)
else:
    raise SystemExit("not refused")
print("ok")
"""


def test_library_loads_without_the_calls_module():
    r = subprocess.run([sys.executable, "-c", WITHOUT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stderr[-2000:]
