"""Builds libsurgeon.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsurgeon.so")
# the checked build: every guarded global store tests its index (-DSURGEON_BOUNDS)
LIB_BOUNDS = os.path.join(HERE, "libsurgeon_bounds.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared", "--use_fast_math=false",
]


# the marshalling of short calls (a Python module that only passes arguments on)
CALLS = os.path.join(HERE, "_calls.so")
CALLS_SOURCE = os.path.join(HERE, "pyext", "calls.cpp")


def build_calls(force: bool = False) -> str:
    """Builds _calls.so with g++ against the installed PyTorch."""
    import sysconfig

    import torch
    deps = [CALLS_SOURCE, os.path.join(ROOT, "include", "surgeon.h")]
    if not force and os.path.exists(CALLS) and all(os.path.getmtime(p) <= os.path.getmtime(CALLS) for p in deps):
        return CALLS
    at = os.path.dirname(torch.__file__)
    include = [os.path.join(ROOT, "include"), os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    tmp = CALLS + ".tmp%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch.compiled_with_cxx11_abi())]
                          + [a for p in include for a in ("-I", p)] + [CALLS_SOURCE, "-o", tmp, "-L", os.path.join(at, "lib")]
                          + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])
    os.replace(tmp, CALLS)
    return CALLS


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(
        os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False, bounds: bool = False) -> str:
    lib = LIB_BOUNDS if bounds else LIB
    if not force and not needs_build(lib):
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = [f for f in NVCC_FLAGS if not f.startswith("--use_fast_math")]
    if verbose:
        flags += ["-Xptxas", "-v"]
    if bounds:
        flags += ["-DSURGEON_BOUNDS"]
    tmp = lib + ".tmp%d" % os.getpid()
    cmd = [nvcc] + flags + ["-I", os.path.join(ROOT, "include"), "-I", CSRC] + sources() + [
        "-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    build_calls(force="--force" in sys.argv)
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, bounds="--bounds" in sys.argv))
