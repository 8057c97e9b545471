"""The very first call on a device, made while a stream is being captured: each entry point in a process of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

COMMON = """
import torch
import paper_2510_08431_b200 as aj
g = torch.Generator(device="cuda").manual_seed(3)
rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
q, k, v, tq, tk, tv, d_o = (rn(1, 300, 2, 64) for _ in range(7))
x, h = rn(2, 40, 128), rn(2, 40, 128)
mask = torch.rand(1, 2, 3, 3, generator=g, device="cuda") < 0.6
layer, core, dense = aj.AdaLNJVP(128), aj.SparseAttentionCoreJVP(2), aj.AttentionCoreJVP()

def step():
    %s

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in got]
want = step()
torch.cuda.synchronize()
assert aj.attn_jvp_device_status() == 0
for a, b in zip(got, want):
    assert torch.equal(a, b)
print("same")
"""
STEPS = dict(
    dense="return aj.attention_jvp(q, k, v, tq, tk, tv)",
    dense_forward="return dense(q, k, v),",
    sparse_forward="s = aj.block_selection(mask, 300, 300); return aj.sparse_attention_jvp(q, k, v, s, tq, tk, tv)",
    sparse_training="s = aj.block_select(q, k, 2); o, _, l = aj.sparse_attention_jvp(q, k, v, s, fwd_only=True); "
                    "return aj.sparse_attention_backward(d_o, q, k, v, o, l, s)",
    sparse_backward="s = aj.block_selection(mask, 300, 300); l = torch.zeros(1, 2, 300, device='cuda') + 5; "
                    "return aj.sparse_attention_backward(d_o, q, k, v, q, l, s)",
    layer="return core(q, k, v),",
    adaln="return (*layer(x, h), *aj.adaln_backward(x, h, x, h)[:2])",
    qknorm="return aj.qknorm_jvp(q, tq, torch.ones(64, device='cuda'))",
)


@pytest.mark.parametrize("name", STEPS)
def test_first_call_inside_a_capture(name):
    code = COMMON % STEPS[name]
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=180)
    assert res.returncode == 0 and res.stdout.strip() == "same", res.stderr[-3000:]
