"""How far a value that is not finite reaches under a causal mask: what sees it, and at most the rest of the 128 x 128 blocks that the mask cuts."""
import pytest
import torch

from tests.test_gpu_attention import aj, inputs, no_timeout  # noqa: F401

pytestmark = pytest.mark.gpu


def run(aj, x):
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, causal=True)
    dq, dk, dv = aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, causal=True)
    _, to, _ = aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], x["tk"], x["tv"], causal=True)
    no_timeout(aj)
    return dict(o=o, to=to, dq=dq, dk=dk, dv=dv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", ["q", "k", "v", "d_o"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("Lq,Lk", [(600, 600), (400, 670)])
def test_reach(aj, D, name, bad, Lq, Lk):
    x = inputs(1, 2, 2, Lq, Lk, D)
    clean = run(aj, x)
    at, off = 333, Lk - Lq
    y = dict(x, **{name: x[name].clone()})
    y[name][0, at, 1] = bad
    got = run(aj, y)
    query, key = torch.arange(Lq, device="cuda")[:, None], torch.arange(Lk, device="cuda")
    seen = key <= query + off
    # a block is reached if any of its pairs is seen
    blocks = torch.zeros(-(-Lq // 128) * 128, -(-Lk // 128) * 128, dtype=torch.bool, device="cuda")
    blocks[:Lq, :Lk] = seen
    blocks = blocks.unflatten(0, (-1, 128)).unflatten(2, (-1, 128)).any(3).any(1).repeat_interleave(128, 0).repeat_interleave(128, 1)[:Lq, :Lk]
    if name in ("q", "d_o"):                             # a query: its own row, and the keys that its block meets
        row = torch.zeros(Lq, dtype=torch.bool, device="cuda")
        row[at] = True
        rows = {n: row if n in ("o", "to", "dq") else blocks[at] for n in got}
    else:                                                # a key: its own gradients and the queries that its block meets; their delta reaches on in dK
        rows = {n: blocks[:, at] if n in ("o", "to", "dq") else torch.ones(Lk, dtype=torch.bool, device="cuda") for n in got}
    for n, may in rows.items():
        assert torch.equal(got[n][:, ~may], clean[n][:, ~may]), n
        assert torch.equal(got[n][:, :, 0], clean[n][:, :, 0]), n            # (the other head)
    if name in ("k", "v"):                               # who sees it shows it
        assert not torch.isfinite(got["dq" if name == "k" else "o"][0, seen[:, at], 1]).all(-1).any()
    else:
        assert not torch.isfinite(got["dk"][0, seen[at], 1]).all(-1).any()
