"""What the host binding does besides checking its arguments."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

OUT_OF_MEMORY = """
import torch
import paper_2510_08431_b200 as aj
x = torch.randn(1, 60000, 1024, device="cuda").bfloat16()
q = x.view(1, 60000, 8, 128)
torch.cuda.empty_cache()                 # (or the selection would lie in a large free block and keep it)
sel = aj.block_select(q, q, 1)
calls = (lambda: aj.adaln_jvp(x), lambda: aj.adaln_backward(x, x, x), lambda: aj.sparse_attention_jvp(q, q, q, sel, fwd_only=True),
         lambda: aj.attention_jvp(q, q, q, fwd_only=True))
torch.cuda.synchronize()
torch.cuda.empty_cache()
total = torch.cuda.mem_get_info()[1]
torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (8 << 20)) / total)
raised = 0
for call in calls:
    try:
        call()
    except torch.OutOfMemoryError:
        raised += 1
torch.cuda.set_per_process_memory_fraction(1.0)
for call in calls:
    call()
torch.cuda.synchronize()
assert aj.attn_jvp_device_status() == 0
print(raised, "of", len(calls))
"""


def test_out_of_memory_is_the_error_that_torch_raises():
    """A caller that makes its batch smaller on torch.OutOfMemoryError can do so here too; the calls work again afterwards."""
    res = subprocess.run([sys.executable, "-c", OUT_OF_MEMORY], cwd=ROOT, capture_output=True, text=True, timeout=180)
    assert res.returncode == 0 and res.stdout.strip() == "4 of 4", res.stdout + res.stderr[-3000:]
