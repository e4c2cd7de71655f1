"""Builds ``libdeepcache.so`` in-tree with nvcc for sm_100a, and ``_tensors.so``, its binding to torch tensors, with the C++ compiler."""
from __future__ import annotations

import glob
import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(_HERE), "include")
LIB = os.path.join(_HERE, "libdeepcache.so")
TENSORS = os.path.join(_HERE, "_tensors.so")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_and_python() -> str:
    """What ``_tensors.so`` is made for.  It holds this text itself, so that it is made anew when one of the two changes."""
    import sys
    import torch
    return f"_tensors for torch {torch.__version__}, python {sys.version_info.major}.{sys.version_info.minor}"


def tensors_command():
    """How ``_tensors.so`` is made: torch's own headers and libraries, libdeepcache found beside it."""
    import sysconfig
    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    includes = [sysconfig.get_paths()["include"], INCLUDE, *cpp_extension.include_paths(), os.path.join(cuda, "include")]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            f'-DDC_BUILT_FOR="{_torch_and_python()}"',
            *(f for i in includes for f in ("-isystem" if "torch" in i else "-I", i)), os.path.join(CSRC, "dc_torch.cpp"), "-o", TENSORS,
            "-L", libs, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-L", _HERE, "-ldeepcache", "-Wl,-rpath,$ORIGIN"]


def tensors_stale() -> bool:
    if not os.path.exists(TENSORS):
        return True
    t = os.path.getmtime(TENSORS)
    if any(os.path.getmtime(d) > t for d in (os.path.join(CSRC, "dc_torch.cpp"), os.path.join(INCLUDE, "deepcache.h"))):
        return True
    with open(TENSORS, "rb") as f:
        return _torch_and_python().encode() + b"\0" not in f.read()


def tensors_lack() -> str:
    """What ``_tensors.so`` needs beside nvcc and is not there, or an empty text."""
    import importlib.util
    import shutil
    import sysconfig
    if importlib.util.find_spec("torch") is None:
        return "torch"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python's headers"
    cxx = os.environ.get("CXX", "g++")
    return "" if shutil.which(cxx) else f"the C++ compiler {cxx}"


def build_tensors(force: bool = False) -> str:
    if force or tensors_stale():
        subprocess.check_call(tensors_command())
    return TENSORS


def build(force: bool = False, verbose: bool = False) -> str:
    """Both libraries.  The C library needs nvcc alone; where what the binding to torch tensors needs is not there, it is left out and that is
    said, and its calls say so in their turn."""
    build_library(force, verbose)
    lack = tensors_lack()
    if lack:
        print(f"{os.path.basename(TENSORS)} is not built: {lack} is missing")
    else:
        build_tensors(force)
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    objs = []
    build_dir = os.path.join(_HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    procs = []
    for src in sources():
        obj = os.path.join(build_dir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [nvcc, *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC,
               "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            print(f"--- {os.path.basename(src)}\n{out}")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call([nvcc, "-shared", "-o", LIB, *objs, "-lcudart"])
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
