"""The C++ calls module is bound by the paged functions alone: SubGen and the exact cache do without it."""
import os
import shutil
import subprocess
import sys

import pytest

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


def test_another_torch_makes_the_module_stale(monkeypatch, tmp_path):
    """However new the file is: an update of torch leaves the sources' times as they are."""
    import torch
    from paper_2402_06082_b200 import build
    build.build()
    assert not build._calls_stale()
    copy = str(tmp_path / "_calls.so")
    shutil.copy(build.CALLS, copy)
    monkeypatch.setattr(build, "CALLS", copy)
    assert not build._calls_stale()
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".1")
    assert build._calls_stale()
    monkeypatch.undo()
    monkeypatch.setattr(build, "CALLS", copy)
    os.remove(copy)
    assert build._calls_stale()


def test_a_module_for_another_torch_is_refused(monkeypatch):
    import torch
    from paper_2402_06082_b200 import binding
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.setattr(torch, "__version__", "0.0")
    with pytest.raises(RuntimeError, match="built for"):
        binding.qk_norm_rope(torch.zeros(1, 1, 64), None)
    monkeypatch.undo()
    with pytest.raises(ValueError):
        binding.qk_norm_rope(torch.zeros(1, 1, 64), None)
