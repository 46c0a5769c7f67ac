"""Compile the HIP sources under csrc/ into libsasgd.so for gfx950 and the CPython module beside it (run: python -m paper_1511_05950_amd.build)."""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsasgd.so")
PYEXT_SRC = os.path.join(HERE, "pyext", "fastcalls.c")
PYEXT = os.path.join(HERE, "_fastcalls.so")

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-x", "hip",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-warning-option",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def build(force=True, verbose=False):
    """Compile every source and link libsasgd.so.  force=False skips up-to-date objects."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ, exist_ok=True)
    headers = glob.glob(os.path.join(CSRC, "*.hpp")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)

    def compile_one(src):
        obj = os.path.join(OBJ, os.path.basename(src) + ".o")
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(src), newest_header):
            return obj
        cmd = [hipcc] + FLAGS + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed on %s:\n%s" % (src, err))
        if err.strip() and verbose:
            print(err, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, sources()))
    cmd = [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    build_pyext()
    return LIB


# What fastcalls.c uses of torch's C interface to its tensors.
TENSOR_PROBE = """
#include <ATen/dlpack.h>
int usable(const DLPackExchangeAPI* a, void* o, DLTensor* t) {
  return a->header.version.major == DLPACK_MAJOR_VERSION && a->dltensor_from_py_object_no_sync && a->dltensor_from_py_object_no_sync(o, t) == 0 &&
         t->device.device_type != kDLCUDA && t->device.device_type != kDLROCM && t->dtype.code == kDLBfloat;
}
"""


def tensor_flags():
    """Compiler flags that let the module read tensors through torch's C interface; none where this torch has no such headers, or there is none (it then
    reads them through their methods)."""
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.origin:
        return []
    flags = ["-DSASGD_TORCH_TENSORS", "-I", os.path.join(os.path.dirname(spec.origin), "include")]
    r = subprocess.run([os.environ.get("CC", "gcc"), "-std=c11", "-fsyntax-only", *flags, "-x", "c", "-"], input=TENSOR_PROBE, capture_output=True, text=True)
    return flags if r.returncode == 0 else []


def build_pyext():
    """The CPython module of the per-gradient and per-update calls (host code only), linked against libsasgd.so beside it."""
    cmd = [os.environ.get("CC", "gcc"), "-O2", "-std=c11", "-fPIC", "-shared", "-Wall", "-I", sysconfig.get_paths()["include"], *tensor_flags(), PYEXT_SRC, "-o", PYEXT,
           "-L", HERE, "-l:libsasgd.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("building %s failed:\n%s" % (PYEXT, r.stderr))


if __name__ == "__main__":
    print(build(force="--incremental" not in sys.argv, verbose=True))
