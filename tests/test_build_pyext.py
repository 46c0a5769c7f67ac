"""The CPython module builds with the torch that is there, with one whose headers do not offer its tensors in C, and with none; the calls are the same."""
import importlib.util
import os
import subprocess
import sys

import pytest

from paper_1511_05950_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# one tensor of each kind through list_of's checks, on the host (device -1): what is wrong with it is refused before the library is called
CHECKS = """
import sys, importlib.util
sys.path.insert(0, sys.argv[2])
import torch
from paper_1511_05950_amd import binding as b
b.load()
spec = importlib.util.spec_from_file_location("_fastcalls", sys.argv[1])
fast = importlib.util.module_from_spec(spec)
spec.loader.exec_module(fast)
fast.set_error_class(b.SasgdError)
for one in (fast, b._fast):
    one.set_tensor_class(torch.Tensor, torch.float32, torch.bfloat16)
out, work = torch.zeros(2), torch.zeros(b.NORM_WORKSPACE, dtype=torch.uint8)
for grads, error in (([torch.zeros(4, dtype=torch.float64)], TypeError), ([torch.zeros(8)[::2]], ValueError), ([torch.zeros(4), torch.zeros(4).bfloat16()], TypeError),
                     ([torch.zeros(4, 4).t()], ValueError)):
    try:
        fast.gradient_norm(grads, 0.0, out, work, -1, 0)
        raise SystemExit("not refused")
    except error:
        pass
assert fast.group_norm_workspace(torch.zeros(2, 8, 8, 32), 4, 1) == b._fast.group_norm_workspace(torch.zeros(2, 8, 8, 32), 4, 1) > 0
print("same")
"""


@pytest.mark.parametrize("torch_is", ["there", "old", "without headers", "absent"])
def test_module_builds_and_checks(torch_is, tmp_path, monkeypatch):
    found = importlib.util.find_spec
    if torch_is == "old":
        (tmp_path / "torch" / "include" / "ATen").mkdir(parents=True)
        (tmp_path / "torch" / "include" / "ATen" / "dlpack.h").write_text("typedef struct { int ndim; } DLTensor;\n")
    spec = {"old": importlib.util.spec_from_file_location("torch", str(tmp_path / "torch" / "__init__.py")),
            "without headers": importlib.util.spec_from_file_location("torch", str(tmp_path / "nowhere" / "torch" / "__init__.py")), "absent": None}
    if torch_is in spec:
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: spec[torch_is] if name == "torch" else found(name, *a))
    module = str(tmp_path / "_fastcalls.so")
    monkeypatch.setattr(build, "PYEXT", module)
    build.build_pyext()
    script = tmp_path / "checks.py"
    script.write_text(CHECKS)
    # (linked for a library beside it)
    os.symlink(build.LIB, str(tmp_path / "libsasgd.so"))
    r = subprocess.run([sys.executable, str(script), module, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr
