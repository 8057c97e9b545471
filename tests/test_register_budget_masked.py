"""What the compiler says about the attention kernels with a mask and the gradients' kernels (nvcc alone, no GPU)."""
import re
import subprocess

import pytest

from paper_2510_08431_b200 import build

# <D, mode, softmax groups>: spill loads in bytes.  Built with CUDA 12.9 they are 84, 84, 228 and 244, 332, 192.
MASKED = [(64, "kModeJvp", 2, 95), (64, "kModeKvTangentFree", 2, 95), (64, "kModeFwdOnly", 2, 250),
          (128, "kModeJvp", 1, 270), (128, "kModeKvTangentFree", 1, 365), (128, "kModeFwdOnly", 2, 210)]
GRADIENTS = [(64, True), (64, False), (128, True), (128, False)]         # <D, pass>: registers are dealt out to the warps by hand, nothing spills


@pytest.fixture(scope="module")
def spills(tmp_path_factory):
    """{kernel's mangled name: bytes of spill loads}."""
    d = tmp_path_factory.mktemp("ptxas")
    src = d / "kernels.cu"
    names = [f"attn_jvp::attn_jvp_fwd_kernel<{D}, attn_jvp::{mode}, false, {groups}, false, false, true>" for D, mode, groups, _ in MASKED]
    names += [f"attn_jvp::dense_bwd_kernel<{D}, {str(dkv).lower()}>" for D, dkv in GRADIENTS]
    table = ", ".join(f"reinterpret_cast<const void*>({n})" for n in names)
    src.write_text(f'#include "dense_bwd.cuh"\nextern const void* const kernels[];\nconst void* const kernels[] = {{{table}}};\n')
    csrc = build.SRC.rsplit("/", 1)[0]
    res = subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-cubin", "-Xptxas", "-v",
                          "-I", csrc, "-o", str(d / "kernels.cubin"), str(src)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return {n: int(loads) for n, loads in re.findall(r"Function properties for (\w+)\s+\d+ bytes stack frame, \d+ bytes spill stores, (\d+) bytes spill loads", res.stderr)}


@pytest.mark.parametrize("D,mode,groups,most", MASKED)
def test_masked_attention(spills, D, mode, groups, most):
    m = {"kModeJvp": 0, "kModeKvTangentFree": 1, "kModeFwdOnly": 2}[mode]
    (loads,) = [v for n, v in spills.items() if f"attn_jvp_fwd_kernelILi{D}ELi{m}ELb0ELi{groups}ELb0ELb0ELb1E" in n]
    assert loads <= most, f"{loads} bytes of spill loads"


@pytest.mark.parametrize("D,dkv", GRADIENTS)
def test_gradients(spills, D, dkv):
    (loads,) = [v for n, v in spills.items() if f"dense_bwd_kernelILi{D}ELb{int(dkv)}E" in n]
    assert loads == 0, f"{loads} bytes of spill loads"
