"""The three directions of the fused gate + residual + norm + modulation step, twice: 12000 tokens x 5120 channels, bf16, layer norm."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_08431_b200 as aj  # noqa: E402

L, C = 12000, 5120
x, h, tx, th, dx, dy = (torch.randn(1, L, C, device="cuda").bfloat16() for _ in range(6))
gate, scale, shift = torch.randn(1, 3, C, device="cuda").unbind(1)
for _ in range(2):
    aj.adaln_jvp(x, h, gate, scale, shift)
    aj.adaln_jvp(x, h, gate, scale, shift, tx=tx, th=th, tgate=gate, tscale=scale, tshift=shift)
    aj.adaln_backward(dx, dy, x, h, gate, scale, shift)
torch.cuda.synchronize()
print("ok")
