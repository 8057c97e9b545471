"""Builds libattn_jvp.so (sm_100a only) in-tree with nvcc.  Needs no GPU."""
from __future__ import annotations

import os
import shutil
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "attn_jvp.cu")
DEPS = [SRC, os.path.join(PKG, "csrc", "attn_jvp_kernel.cuh"), os.path.join(PKG, "csrc", "qknorm_jvp.cuh"),
        os.path.join(PKG, "csrc", "adaln_jvp.cuh"), os.path.join(PKG, "csrc", "block_select.cuh"),
        os.path.join(PKG, "csrc", "sparse_bwd.cuh"),
        os.path.join(ROOT, "include", "attn_jvp.h")]
LIB = os.path.join(PKG, "libattn_jvp.so")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the attention-JVP library is CUDA-only (sm_100a) and has no fallback")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in DEPS)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if it is missing or older than its sources; returns its path."""
    if not force and not is_stale():
        return LIB
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
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
