"""As tests/test_gpu_first_call_captured.py, for the rotary calls and dense attention in training."""
import subprocess
import sys

import pytest

from tests.test_gpu_first_call_captured import COMMON, ROOT

pytestmark = pytest.mark.gpu
STEPS = dict(
    table="return aj.rotary_table(q[0, :, 0, 0].float(), 64),",
    rotary="t = torch.ones(300, 16, 2, device='cuda'); w = torch.ones(64, device='cuda'); "
           "return (*aj.qk_rotary_jvp(q, k, t, tq=tq, tk=tk), *aj.qk_rotary_backward(q, k, q, k, t, norm='rms', q_weight=w, k_weight=w)[:4])",
    masked="n = torch.full((1,), 170, dtype=torch.int32, device='cuda'); return aj.attention_jvp(q, k, v, tq, tk, tv, causal=True, k_lengths=n)",
    backward="l = torch.zeros(1, 2, 300, device='cuda') + 5; return aj.attention_backward(d_o, q, k, v, q, l)",
    training="o, _, l = aj.attention_jvp(q, k[:, :, :1], v[:, :, :1], fwd_only=True, causal=True); "
             "return aj.attention_backward(d_o, q, k[:, :, :1], v[:, :, :1], o, l, causal=True)",
)


@pytest.mark.parametrize("name", STEPS)
def test_first_call_inside_a_capture(name):
    res = subprocess.run([sys.executable, "-c", COMMON % STEPS[name]], cwd=ROOT, capture_output=True, text=True, timeout=180)
    assert res.returncode == 0 and res.stdout.strip() == "same", res.stderr[-3000:]
