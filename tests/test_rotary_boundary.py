"""Argument checks of the rotary calls at the C ABI (no GPU work), and pins of their 64-bit statement."""
import math

import pytest
import torch

from tests import rotary_ref as R

A, STEP = 0x7F0000000000, 1 << 33        # fake, aligned, well separated addresses


@pytest.fixture(scope="module")
def aj():
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def table(aj, positions=A, pos_type=2, n=10, dims=(64,), base=(1e4,), scaling=0, factor=(1.0,), original_length=0.0, out=A + STEP):
    return aj.attn_jvp_rotary_table(positions, pos_type, n, dims, base, scaling, factor, original_length, out, None)


def test_table_refuses(aj):
    for kw in (dict(positions=None), dict(out=None)):
        assert table(aj, **kw) == 1
    two = dict(base=(1e4, 1e4), factor=(1.0, 1.0))
    for kw in (dict(n=0), dict(dims=(3,)), dict(dims=(0,)), dict(dims=(258,)), dict(dims=(128, 130), **two), dict(dims=(64, 2), scaling=2, **two)):
        assert table(aj, **kw) == 2
    for kw in (dict(pos_type=0), dict(pos_type=7), dict(scaling=4), dict(scaling=-1)):
        assert table(aj, **kw) == 5
    for kw in (dict(base=(0.0,)), dict(base=(math.nan,)), dict(factor=(-1.0,)), dict(factor=(math.inf,)), dict(scaling=3, original_length=0.0)):
        assert table(aj, **kw) == 6
    assert table(aj, positions=A + 2) == 4 and table(aj, pos_type=3, positions=A + 4) == 4 and table(aj, out=A + STEP + 8) == 4
    assert table(aj, out=A) == 7


def args(aj, **kw):
    a = aj.QKRotaryArgs()
    names = ("q", "k", "tq", "tk", "q_weight", "k_weight", "q_bias", "k_bias", "table", "index")
    for i, n in enumerate(names):
        setattr(a, n, A + i * STEP)
    v = dict(B=2, L=30, H=4, Hk=2, D=64, R=32, norm=2, layout=0, eps=1e-6, table_rows=30, table_batch=0, index_batch=30)
    v.update(kw)
    strides = v.pop("strides", {})
    for n, h in (("q", v["H"]), ("k", v["Hk"]), ("tq", v["H"]), ("tk", v["Hk"])):
        s = strides.get(n, (v["L"] * h * v["D"], h * v["D"], v["D"]))
        getattr(a, n + "_stride")[:] = [max(-(1 << 62), min(1 << 62, t)) for t in s]
    for n, t in v.items():
        setattr(a, n, t)
    return a


def fwd(aj, q=A + 20 * STEP, k=A + 21 * STEP, tq=A + 22 * STEP, tk=A + 23 * STEP, **kw):
    return aj.attn_jvp_qk_rotary_fwd(args(aj, **kw), q, k, tq, tk, None)


def bwd(aj, dqn=A + 20 * STEP, dkn=A + 21 * STEP, dq=A + 22 * STEP, dk=A + 23 * STEP, dw=(A + 24 * STEP, A + 25 * STEP, A + 26 * STEP, A + 27 * STEP),
        ws=A + 28 * STEP, n=1 << 30, **kw):
    return aj.attn_jvp_qk_rotary_bwd(args(aj, **kw), dqn, dkn, dq, dk, *dw, ws, n, None)


def test_heads_refuse(aj):
    for call in (fwd, bwd):
        for kw in (dict(B=0), dict(L=0), dict(H=0), dict(R=0), dict(R=12), dict(R=72), dict(B=1 << 15, L=1 << 15), dict(table_rows=0),
                   dict(table_batch=-1), dict(index=None, table_rows=29), dict(strides=dict(q=(4, 256, 64))), dict(strides=dict(k=(1 << 12, -128, 64)))):
            assert call(aj, **kw) == 2, kw
        assert call(aj, D=96) == 3
        assert call(aj, norm=3) == 5 and call(aj, layout=2) == 5 and call(aj, eps=-1.0) == 6 and call(aj, eps=math.inf) == 6
        assert call(aj, q=A + 8) == 4 if call is bwd else True
        assert call(aj, table=A + 8 * STEP + 8) == 4 and call(aj, q_weight=A + 2) == 4 and call(aj, index=A + 2) == 4
    for kw in (dict(q=None), dict(k=None), dict(tq=None), dict(tk=None)):
        assert fwd(aj, **kw) == 1
    assert aj.attn_jvp_qk_rotary_fwd(args(aj, q=None), A + 20 * STEP, A + 21 * STEP, None, None, None) == 1
    assert aj.attn_jvp_qk_rotary_fwd(args(aj, table=None), A + 20 * STEP, A + 21 * STEP, None, None, None) == 1
    assert aj.attn_jvp_qk_rotary_fwd(args(aj, k=None), A + 20 * STEP, None, None, None, None) == 1       # (Hk says 2)
    assert fwd(aj, q=A + 20 * STEP + 8) == 4 and fwd(aj, q=A) == 7 and fwd(aj, tk=A + 22 * STEP) == 7 and fwd(aj, k=A + 9 * STEP) == 7
    for kw in (dict(dqn=None), dict(dkn=None), dict(dq=None), dict(dk=None), dict(ws=None)):
        assert bwd(aj, **kw) == 1
    need = aj.attn_jvp_qk_rotary_bwd_workspace_bytes(2, 30, 4, 2, 64)
    assert need > 0 and bwd(aj, n=need - 1) == 12 and bwd(aj, ws=A + 28 * STEP + 8) == 4 and bwd(aj, dq=A) == 7 and bwd(aj, ws=A + 24 * STEP) == 7
    for bad in ((0, 1, 1, 1, 64), (1, 1, 0, 1, 64), (1, 1, 1, -1, 64), (1, 1, 1, 1, 96), (1 << 16, 1 << 16, 1, 1, 64)):
        assert aj.attn_jvp_qk_rotary_bwd_workspace_bytes(*bad) == 0


def test_statement():
    """Rotations keep lengths and depend on differences of positions alone; a position of 0 changes nothing; pairs as named."""
    g = torch.Generator().manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x, y = rn(1, 1, 1, 8), rn(1, 1, 1, 8)
    t = R.table(torch.arange(50).view(1, 50, 1), (8,))
    for layout in ("interleaved", "half"):
        at = lambda v, p: R.turn(v, t[:, p:p + 1], layout)
        assert torch.allclose(at(x, 0), x) and torch.allclose(at(x, 37).norm(), x.norm())
        assert torch.allclose((at(x, 12) * at(y, 5)).sum(), (at(x, 40) * at(y, 33)).sum())
    one = torch.zeros(1, 1, 1, 8, dtype=torch.float64)
    one[..., 0] = 1
    c, s = math.cos(3), math.sin(3)                                  # (the first pair turns one radian per position)
    a, b = R.turn(one, t[:, 3:4], "interleaved")[0, 0, 0], R.turn(one, t[:, 3:4], "half")[0, 0, 0]
    assert abs(a[0] - c) < 1e-12 and abs(a[1] - s) < 1e-12 and abs(b[0] - c) < 1e-12 and abs(b[4] - s) < 1e-12
    # the stretched tables: linear at factor s is the plain one at position / s; the slowest ntk pair too; yarn keeps the fast pairs
    pos = torch.arange(40).view(40, 1)
    plain = R.table(pos.double() / 4, (16,))
    assert torch.allclose(R.table(pos, (16,), scaling="linear", factor=4.0), plain)
    assert torch.allclose(R.table(pos, (16,), scaling="ntk", factor=4.0)[:, -1], plain[:, -1])
    m = 0.1 * math.log(4) + 1
    yarn = R.table(pos, (16,), scaling="yarn", factor=4.0, original_length=4096)
    assert torch.allclose(yarn[:, 0], m * R.table(pos, (16,))[:, 0])
    slow = R.table(pos, (16,), scaling="yarn", factor=4.0, original_length=6)      # (under one turn: every pair is stretched)
    assert torch.allclose(slow, m * plain)
