"""Selection, forward and gradients of attention over selected key blocks, twice: four heads of 18944 tokens (148 blocks), D = 128, 32 key
blocks per query block."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_08431_b200 as aj  # noqa: E402

q, k, v, d_o = (torch.randn(1, 18944, 4, 128, device="cuda").bfloat16() for _ in range(4))
for _ in range(2):
    sel = aj.block_select(q, k, 32)
    o, _, lse = aj.sparse_attention_jvp(q, k, v, sel, fwd_only=True)
    aj.sparse_attention_backward(d_o, q, k, v, o, lse, sel)
torch.cuda.synchronize()
assert aj.attn_jvp_device_status() == 0
print("ok")
