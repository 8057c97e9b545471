"""Argument checks of the masked attention calls at the C ABI (no GPU work), and pins of their 64-bit statement."""
import math

import pytest
import torch

from tests import attention_ref as R
from tests import sparse_ref

A, STEP = 0x7F0000000000, 1 << 33        # fake, aligned, well separated addresses
BASE = dict(B=2, H=4, Hk=2, Lq=300, Lk=500, D=64)


@pytest.fixture(scope="module")
def aj():
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def args(aj, **kw):
    a = aj.AttentionArgs()
    for i, n in enumerate(("q", "k", "v", "tq", "tk", "tv", "k_lengths")):
        setattr(a, n, A + i * STEP)
    v = dict(**BASE, causal=0, scale=0.1)
    v.update(kw)
    for n, h, L in (("q", v["H"], v["Lq"]), ("k", v["Hk"], v["Lk"]), ("v", v["Hk"], v["Lk"])):
        s = v.pop(n + "_stride", (L * h * v["D"], h * v["D"], v["D"]))
        getattr(a, n + "_stride")[:] = [max(-(1 << 62), min(1 << 62, t)) for t in s]
    for n, t in v.items():
        setattr(a, n, t)
    return a


def fwd(aj, o=A + 8 * STEP, to=A + 9 * STEP, lse=A + 10 * STEP, mu=A + 11 * STEP, flags=0, **kw):
    return aj.attn_jvp_attention_fwd(args(aj, **kw), o, to, lse, mu, flags, None)


def bwd(aj, d_o=A + 8 * STEP, o=A + 9 * STEP, lse=A + 10 * STEP, dq=A + 11 * STEP, dk=A + 12 * STEP, dv=A + 13 * STEP, ws=A + 14 * STEP, n=1 << 32, **kw):
    return aj.attn_jvp_attention_bwd(args(aj, **kw), d_o, o, lse, dq, dk, dv, ws, n, None)


def test_refusals(aj):
    for call in (fwd, bwd):
        for kw in (dict(B=0), dict(H=0), dict(Hk=0), dict(Hk=3), dict(H=2, Hk=4), dict(Lq=0), dict(Lk=-1), dict(Lk=786433), dict(B=70000), dict(H=1 << 30, Hk=1),
                   dict(q_stride=(76800, 256, 4)), dict(q_stride=(76800, 0, 64)), dict(k_stride=(-64, 128, 64)), dict(v_stride=(1 << 50, 128, 64)), dict(k_stride=(64000, 128, 32))):
            assert call(aj, **kw) == 2, kw
        assert call(aj, D=96) == 3 and call(aj, scale=math.nan) == 6 and call(aj, causal=2) == 5
        for n in ("q", "k", "v"):
            assert call(aj, **{n: None}) == 1
        assert call(aj, q=A + 8) == 4 and call(aj, k_lengths=A + 2) == 4 and call(aj, lse=A + 10 * STEP + 2) == 4
    for n in ("o", "to", "lse", "tq", "tk", "tv"):
        assert fwd(aj, **{n: None}) == 1
    assert fwd(aj, flags=4) == 5 and fwd(aj, o=A) == 7 and fwd(aj, to=A + 8 * STEP) == 7 and fwd(aj, mu=A + 6 * STEP) == 7
    for n in ("d_o", "o", "lse", "dq", "dk", "dv", "ws"):
        assert bwd(aj, **{n: None}) == 1
    need = aj.attn_jvp_attention_bwd_workspace_bytes(**BASE)
    assert need > 0 and bwd(aj, n=need - 1) == 12 and bwd(aj, ws=A + 14 * STEP + 128) == 4 and bwd(aj, dq=A + STEP) == 7 and bwd(aj, dk=A + 13 * STEP) == 7
    for bad in (dict(B=0), dict(Hk=3), dict(D=96), dict(Lq=0), dict(Hk=0)):
        assert aj.attn_jvp_attention_bwd_workspace_bytes(**{**BASE, **bad}) == 0


def test_workspace_stays_in_proportion(aj):
    """Parts only where there are few blocks: the sums take a few hundred MB at most, and nothing at video length."""
    assert aj.attn_jvp_attention_bwd_workspace_bytes(1, 40, 40, 32760, 32760, 128) < 20e6
    for shape in ((1, 1, 1, 786432, 128, 128), (1, 40, 1, 32760, 512, 128), (1, 1, 1, 1, 786432, 64), (3, 16, 16, 8190, 512, 128)):
        assert aj.attn_jvp_attention_bwd_workspace_bytes(*shape) < 600e6, shape


def test_statement():
    """Without masks the sparse statement with every block; shared heads are repeated ones; a length is a shorter sequence; the causal mask against autograd."""
    g = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=g).bfloat16()
    q, k, v, d_o, tq, tk, tv = rn(2, 20, 4, 8), rn(2, 30, 2, 8), rn(2, 30, 2, 8), rn(2, 20, 4, 8), rn(2, 20, 4, 8), rn(2, 30, 2, 8), rn(2, 30, 2, 8)
    wide = lambda t: t.repeat_interleave(2, 2)
    ref = R.attention(q, k, v, 0.3, tq=tq, tk=tk, tv=tv, d_o=d_o)
    sparse = sparse_ref.attention(q, wide(k), wide(v), torch.ones(2, 4, 1, 1, dtype=torch.bool), 0.3, tq, wide(tk), wide(tv), d_o)
    for n in ("o", "lse", "to", "mu", "dq"):
        assert torch.allclose(ref[n][0], sparse[n][0])
    for n in ("dk", "dv"):
        assert torch.allclose(ref[n][0], sparse[n][0].view(2, 30, 2, 2, 8).sum(3))
    short = R.attention(q, k, v, 0.3, lengths=[30, 11], d_o=d_o)
    alone = R.attention(q[1:], k[1:, :11], v[1:, :11], 0.3, d_o=d_o[1:])
    assert torch.allclose(short["o"][0][1], alone["o"][0][0]) and torch.allclose(short["dk"][0][1, :11], alone["dk"][0][0]) and (short["dk"][0][1, 11:] == 0).all()
    leaves = [t.double().requires_grad_() for t in (q, wide(k), wide(v))]
    keep = torch.arange(30) <= torch.arange(20)[:, None] + 10
    S = torch.einsum("bihd,bjhd->bhij", leaves[0], leaves[1]) * 0.3
    O = torch.einsum("bhij,bjhd->bihd", torch.softmax(S.masked_fill(~keep, -math.inf), -1), leaves[2])
    grads = torch.autograd.grad(O, leaves, d_o.double())
    ref = R.attention(q, k, v, 0.3, causal=True, d_o=d_o)
    assert torch.allclose(ref["o"][0], O) and torch.allclose(ref["dq"][0], grads[0]) and torch.allclose(ref["dv"][0], grads[2].view(2, 30, 2, 2, 8).sum(3))
    nothing = R.attention(rn(1, 5, 1, 8), rn(1, 2, 1, 8), rn(1, 2, 1, 8), 1.0, causal=True)
    assert (nothing["lse"][0][0, 0, :3] == -math.inf).all() and (nothing["o"][0][0, :3] == 0).all() and torch.isfinite(nothing["lse"][0][0, 0, 3:]).all()
