"""Tensors that only a call's own sequence holds are alive when the library is called with their addresses (host code only: stand-ins for the library's
functions look, from inside the call)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STAND_INS = """
static void (*look)(void);
void set_look(void (*f)(void)) { look = f; }
int sasgd_gradientNorm(void) { look(); return 0; }
int sasgd_applyAdamW(void) { look(); return 0; }
int sasgd_applyUpdateNoAlloc(void) { look(); return 0; }
"""

CALLS = """
import ctypes, sys, weakref
sys.path.insert(0, sys.argv[2])
stand_ins = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import torch
from paper_1511_05950_amd import binding as b
b.load()
b._fast.set_tensor_class(torch.Tensor, torch.float32, torch.bfloat16)
refs, alive = [], []
look = ctypes.CFUNCTYPE(None)(lambda: alive.append([r() is not None for r in refs]))
stand_ins.set_look(look)

def tensor(kind):
    t = torch.nn.Parameter(torch.zeros(10)) if kind else torch.zeros(10)
    refs.append(weakref.ref(t))
    return t

def check(n, call):
    del refs[:], alive[:]
    call()
    assert alive == [[True] * n], alive
    assert not any(r() is not None for r in refs)          # and not held any longer

out, work = torch.zeros(2), torch.zeros(b.NORM_WORKSPACE, dtype=torch.uint8)
rule = b.SasgdAdamw(0, 0, 0, 0, 1e-3, .9, .9, 1e-8, 0)
tensors = (b.SasgdTensor * 2)(b.SasgdTensor(10, 1, 1, None), b.SasgdTensor(10, 1, 1, None))
moments = b.SasgdMoments(None, None, None, None)
at = [ctypes.addressof(x) for x in (rule, tensors, moments)]
for kind in (0, 1):
    check(3, lambda: b._fast.gradient_norm((tensor(kind) for _ in range(3)), 0.0, out, work, -1, 0))
    check(6, lambda: b._fast.apply_adamw(at[0], at[1], 2, at[2], ((tensor(kind) for _ in range(2)) for _ in range(3)), [0] * 3, 1, None, None, -1, 0))
    check(4, lambda: b._fast.apply_update_no_alloc(0x1000, 0x1000, 0x1000, None, 10, (tensor(kind) for _ in range(4)), [0] * 4, 0, .1, .9, 0., 0))
for bad in ((tensor(0) for _ in range(3)), [[torch.zeros(10), torch.zeros(10)], [torch.zeros(10), torch.zeros(9)]], [(tensor(0) for _ in range(2)), 5]):
    del refs[:], alive[:]
    try:
        b._fast.apply_adamw(at[0], at[1], 2, at[2], bad, [0] * len(bad) if isinstance(bad, list) else [0] * 3, 1, None, None, -1, 0)
        raise SystemExit("not refused")
    except (TypeError, ValueError):
        pass
    assert not alive and not any(r() is not None for r in refs)
print("held")
"""


def test_tensors_of_generators_are_held_until_the_call_returns(tmp_path):
    source, lib, script = tmp_path / "stand_ins.c", tmp_path / "stand_ins.so", tmp_path / "calls.py"
    source.write_text(STAND_INS)
    script.write_text(CALLS)
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", str(lib), str(source)], check=True)
    r = subprocess.run([sys.executable, str(script), str(lib), ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "held" in r.stdout, r.stdout + r.stderr
