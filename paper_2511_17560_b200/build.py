"""Builds, in-tree, liba3.so (the C-ABI CUDA library) with nvcc for sm_100a and a3_calls.so (the compiled part of the Python binding) with g++.

Usage: python -m paper_2511_17560_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "liba3.so")
CALLS = os.path.join(PKG, "a3_calls.so")
CALLS_FOR = os.path.join(PKG, "build", "a3_calls.torch")  # the version of torch that it was made for
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
         "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def calls_stale() -> bool:
    """Whether a3_calls.so is missing, older than its sources, or made for another torch than the one that is installed."""
    import torch

    if _stale(CALLS, [os.path.join(CSRC, "a3_calls.cpp"), os.path.join(ROOT, "include", "a3.h"), os.path.join(os.path.dirname(torch.__file__), "version.py")]):
        return True
    if not os.path.exists(CALLS_FOR):
        return True
    with open(CALLS_FOR) as f:
        return f.read() != str(torch.__version__)


def build_calls(force: bool = False) -> str:
    """a3_calls.so, against the headers and libraries of the torch that is installed."""
    import torch

    src, base = os.path.join(CSRC, "a3_calls.cpp"), os.path.dirname(torch.__file__)
    if force or calls_stale():
        inc = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
               f'-DA3_TORCH_VERSION="{torch.__version__}"',
               "-I", os.path.join(ROOT, "include")] + [a for i in inc for a in ("-isystem", i)]
        cmd += [src, "-o", CALLS, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("g++ failed for " + src)
        os.makedirs(os.path.dirname(CALLS_FOR), exist_ok=True)
        with open(CALLS_FOR, "w") as f:
            f.write(str(torch.__version__))
    return CALLS


def build(force: bool = False, verbose: bool = False) -> str:
    srcs = sources()
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers.append(os.path.join(ROOT, "include", "a3.h"))
    objdir = os.path.join(PKG, "build")
    os.makedirs(objdir, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        if force or _stale(obj, [src] + headers):
            cmd = [NVCC] + FLAGS + extra + ["-c", src, "-o", obj]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if verbose or r.returncode:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode:
                raise RuntimeError("nvcc failed for " + src)
        return obj

    with ThreadPoolExecutor(max_workers=9) as ex:
        calls = ex.submit(build_calls, force)
        objs = list(ex.map(compile_one, srcs))
        calls.result()
    if force or _stale(LIB, objs):
        cmd = [NVCC, "-shared", "-o", LIB] + objs + ["-lcudart", "-lcuda"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("link failed")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
