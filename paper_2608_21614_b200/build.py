"""Builds libsaem.so (the C-ABI CUDA library, nvcc for sm_100a) and _host_calls.so (its inner-loop calls for Python) in-tree.

The library needs nvcc alone; the extension also Python's and torch's headers, and belongs to the Python and the torch that it
was built with.  `binding` builds the one, `mx` and `norms` the other when they are imported."""
from __future__ import annotations

import glob
import importlib
import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libsaem.so")
HOST_LIB = os.path.join(_HERE, "_host_calls.so")
HOST_SOURCE = os.path.join(CSRC, "host_calls.cpp")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
         "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-I", os.path.join(_ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _older(lib, deps) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(p) > t for p in deps)


def _headers():
    return glob.glob(os.path.join(_ROOT, "include", "*.h"))


def stale() -> bool:
    return _older(LIB, sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + _headers())


def _built_for() -> str:
    return "saem_host_calls for Python %s and torch %s" % (sysconfig.get_config_var("SOABI"), importlib.metadata.version("torch"))


def host_stale() -> bool:
    if _older(HOST_LIB, [HOST_SOURCE] + _headers()):
        return True
    with open(HOST_LIB, "rb") as f:
        return (_built_for() + "\0").encode() not in f.read()


def build_host_calls(force: bool = False) -> str:
    """_host_calls.so, linked to the libsaem.so beside it and to torch."""
    if not force and not host_stale():
        return HOST_LIB
    build()
    torch_dir = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.dirname(os.path.dirname(NVCC))
    include = [os.path.join(_ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(torch_dir, "include"),
               os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    tmp = HOST_LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *["-I" + p for p in include],
                           '-DSAEM_BUILT_FOR="%s"' % _built_for(), HOST_SOURCE,
                           "-o", tmp, "-L", os.path.join(torch_dir, "lib"), "-L", _HERE, "-l:" + os.path.basename(LIB), "-ltorch_python",
                           "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, HOST_LIB)
    return HOST_LIB


def host_calls():
    """The module _host_calls, built first if need be (raises if that fails: there is no slower way behind it)."""
    build_host_calls()
    import torch                            # noqa: F401  (brings the libraries that the extension is linked to)
    return importlib.import_module("._host_calls", __package__)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared library (object files in parallel)."""
    if not force and not stale():
        return LIB
    objdir = os.path.join(_HERE, "build")
    os.makedirs(objdir, exist_ok=True)
    procs = []
    objs = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else [])
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode:
            print(out)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    tmp = LIB + ".tmp%d" % os.getpid()
    subprocess.check_call([NVCC, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_host_calls(force="--force" in sys.argv))
