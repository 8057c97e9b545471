"""Builds libattn_jvp.so (sm_100a only) with nvcc and the host binding with g++, in-tree.  Needs no GPU."""
from __future__ import annotations

import os
import shutil
import subprocess
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "attn_jvp.cu")
DEPS = [SRC, os.path.join(PKG, "csrc", "attn_jvp_kernel.cuh"), os.path.join(PKG, "csrc", "qknorm_jvp.cuh"),
        os.path.join(PKG, "csrc", "adaln_jvp.cuh"), os.path.join(PKG, "csrc", "block_select.cuh"),
        os.path.join(PKG, "csrc", "sparse_bwd.cuh"),
        os.path.join(ROOT, "include", "attn_jvp.h")]
LIB = os.path.join(PKG, "libattn_jvp.so")
HOST_SRC = os.path.join(PKG, "csrc", "host_binding.cpp")
HOST_LIB = os.path.join(PKG, "_host.so")
HOST_STAMP = HOST_LIB + ".stamp"         # what the host binding was built against


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the attention-JVP library is CUDA-only (sm_100a) and has no fallback")


def _older(lib: str, deps) -> bool:
    return not os.path.exists(lib) or any(os.path.getmtime(d) > os.path.getmtime(lib) for d in deps)


def is_stale() -> bool:
    return _older(LIB, DEPS)


def _host_stamp() -> str:
    import sys

    import torch
    return f"torch {torch.__version__}, {sys.implementation.cache_tag}"


def host_is_stale() -> bool:
    """The host binding is missing, older than its sources, or of another torch or Python (whose module would not load)."""
    if _older(HOST_LIB, [HOST_SRC, os.path.join(ROOT, "include", "attn_jvp.h")]) or not os.path.exists(HOST_STAMP):
        return True
    with open(HOST_STAMP) as f:
        return f.read() != _host_stamp()


def build_host(force: bool = False) -> str:
    """Compiles the host binding (a CPython module against the installed torch) if it is stale."""
    if not force and not host_is_stale():
        return HOST_LIB
    import sysconfig

    import torch
    tdir = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    includes = [os.path.join(ROOT, "include"), os.path.join(tdir, "include"), os.path.join(tdir, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    tmp = HOST_LIB + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{i}" for i in includes), "-o", tmp, HOST_SRC, f"-L{os.path.join(tdir, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    os.replace(tmp, HOST_LIB)
    with open(tmp, "w") as f:
        f.write(_host_stamp())
    os.replace(tmp, HOST_STAMP)
    return HOST_LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library where it is missing or older than its sources, and after it the host binding; returns the library's path.

    The library needs nvcc alone.  The host binding needs torch's and Python's C++ headers; where it cannot be built, that is a
    warning here, the C ABI and the calls that go through ctypes work, and those that need the binding raise."""
    if force or is_stale():
        _build_library(verbose)
    try:
        build_host(force)
    except (RuntimeError, OSError) as e:
        warnings.warn(f"the host binding is not built, adaln_*, block_sele* and sparse_attention_* will not work: {e}", RuntimeWarning)
    return LIB


def _build_library(verbose: bool) -> None:
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-o", tmp, SRC, "-lcudart"]
    cmd[1:1] = os.environ.get("ATTN_JVP_NVCC_EXTRA", "").split()     # e.g. -DATTN_JVP_DEBUG
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    os.replace(tmp, LIB)
    if verbose:
        print(res.stderr)


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
