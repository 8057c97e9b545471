"""Rotary tables and the per-head norm and rotation of queries and keys against their definitions in 64 bits.

Tolerances.  A bf16 result is off by half a step of its own value (2^-8) and by the fp32 arithmetic before it: some twenty operations, each
off by 2^-24 of the terms that it handles, taken as 2^-19 of the largest such term in the row (`scale`).  Sums of m terms are
off by at most 2^-24 (m' + 20) of the sum of their sizes, m' being the terms that one lane adds one after the other: below 300 at the sizes used here.
"""
import itertools

import pytest
import torch

from tests import rotary_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def close(name, got, want, scale):
    """scale: the size of the terms behind each value, broadcast over rows."""
    off = (got.double() - want).abs()
    most = 2.0 ** -8 * want.abs() + 2.0 ** -19 * scale + 1e-30
    assert torch.isfinite(got).all(), f"{name}: not finite"
    assert (off <= most).all(), f"{name}: {(off / most).max():.3g} of the tolerance"


# ---- tables ----
TABLES = [
    (1, (128,), {}), (777, (2,), {}), (4001, (44, 42, 42), dict(base=(10000.0, 100.0, 500000.0))),
    (1023, (64,), dict(scaling="linear", factor=3.5)), (1023, (64, 32), dict(scaling="ntk", factor=(1.0, 4.0))),
    (5000, (128,), dict(scaling="yarn", factor=8.0, original_length=4096)), (300, (16,) * 8, {}), (70000, (256,), {}),
]


@pytest.mark.parametrize("n,dims,kw", TABLES)
@pytest.mark.parametrize("kind", ["int32", "int64", "fp32"])
def test_table(aj, n, dims, kw, kind):
    g = torch.Generator(device="cuda").manual_seed(n)
    pos = torch.randint(-1000, (1 << 31) - 1 if kind != "fp32" else 5000, (n, len(dims)), generator=g, device="cuda")
    pos = (pos.double() * 0.37).float() if kind == "fp32" else pos.to(dict(int32=torch.int32, int64=torch.int64)[kind])
    got = aj.rotary_table(pos if len(dims) > 1 else pos[:, 0].contiguous(), dims, **kw)
    want = R.table(pos, dims, **kw)
    assert got.shape == want.shape and got.dtype == torch.float32
    # turns are formed to 2^-53 of up to 2^31 / (2 pi) turns, twice (here and in the reference): below 3e-7 radians; then a few roundings of fp32
    far = pos.double().abs().amax() * 2.0 ** -51
    size = want.square().sum(-1).sqrt().amax()
    assert (got.double() - want).abs().max() <= (4 * 2.0 ** -24 + far) * size


def test_table_shapes(aj):
    pos = torch.arange(24, device="cuda", dtype=torch.int32).view(2, 12)
    assert aj.rotary_table(pos, 32).shape == (2, 12, 16, 2)
    assert aj.rotary_table(pos.view(2, 4, 3), (8, 8, 16)).shape == (2, 4, 16, 2)
    assert torch.equal(aj.rotary_table(pos, 32), aj.rotary_table(pos.float(), (32,)))
    for bad in (dict(dims=(3,)), dict(dims=()), dict(dims=(258,)), dict(dims=(8, 8, 8)), dict(dims=(2,), scaling="ntk", factor=2.0),
                dict(dims=(8,), factor=2.0), dict(dims=(8,), scaling="cubic"), dict(dims=(8,), scaling="yarn", factor=2.0),
                dict(dims=(8,), base=-1.0), dict(dims=(8,), scaling="linear", factor=0.0), dict(dims=(8,), base=(1.0, 2.0))):
        with pytest.raises((ValueError, aj.AttnJvpError)):
            aj.rotary_table(pos, **bad)
    for p in (pos.half(), pos.cpu(), pos.T, pos[:0]):
        with pytest.raises((ValueError, aj.AttnJvpError)):
            aj.rotary_table(p, 32)


def test_table_of_no_position(aj):
    """A position that is NaN or infinite has entries of NaN and leaves the others alone."""
    pos = torch.arange(20, device="cuda").float()
    clean = aj.rotary_table(pos, 16)
    pos[3], pos[7], pos[11] = float("nan"), float("inf"), -float("inf")
    got = aj.rotary_table(pos, 16)
    bad = torch.tensor([3, 7, 11], device="cuda")
    assert got[bad].isnan().all() and torch.equal(got[[i for i in range(20) if i not in (3, 7, 11)]], clean[[i for i in range(20) if i not in (3, 7, 11)]])


# ---- heads ----
def inputs(B, L, H, Hk, D, Rt, fused, index, batches, affine, bias, seed=0, rows=None):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * B + L + H)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = {}
    for n in ("", "t"):
        y = (rn(B, L, H + 2 * Hk, D) * torch.exp(0.5 * rn(H + 2 * Hk, D)) + 0.3).bfloat16()
        x[n + "q"], x[n + "k"] = y[:, :, :H], y[:, :, H:H + Hk] if Hk else None
        if not fused:
            x[n + "q"], x[n + "k"] = (None if t is None else t.contiguous() for t in (x[n + "q"], x[n + "k"]))
    x["dq"], x["dk"] = rn(B, L, H, D).bfloat16(), rn(B, L, Hk, D).bfloat16() if Hk else None
    rows = rows or (L + 13 if index else L)
    ang = rn(*((B,) if batches else ()), rows, Rt // 2) * 3
    x["table"] = torch.stack([ang.cos(), ang.sin()], -1)
    x["index"] = None
    if index:
        x["index"] = torch.randint(0, rows, (B, L) if index == 2 else (L,), generator=g, device="cuda").int()
    for n, on in (("q_weight", affine), ("k_weight", affine and Hk), ("q_bias", bias), ("k_bias", bias and Hk)):
        x[n] = (rn(D) * 0.3 + (1 if "w" in n else 0)) if on else None
    return x


CASES = [
    # B, L, H, Hk, D, R, layout, norm, affine, bias, fused, index, batches
    (1, 1, 1, 0, 128, 128, "interleaved", "rms", True, False, False, 0, False),
    (8, 1, 40, 8, 128, 128, "half", "rms", True, False, False, 2, False),
    (2, 333, 5, 1, 128, 128, "interleaved", "rms", True, False, True, 0, True),
    (3, 257, 6, 3, 64, 32, "half", "layer", True, True, True, 0, False),
    (1, 1025, 3, 3, 64, 64, "interleaved", "layer", True, True, False, 1, False),
    (2, 130, 7, 2, 128, 24, "half", None, False, False, True, 2, True),
    (1, 517, 12, 12, 128, 8, "interleaved", None, True, True, False, 0, False),
    (1, 2049, 9, 0, 64, 56, "half", "rms", False, True, True, 0, False),
    (2, 700, 16, 4, 128, 104, "half", "layer", False, False, False, 1, False),
    (1, 4000, 40, 40, 128, 128, "interleaved", "rms", True, False, True, 0, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_heads(aj, case):
    B, L, H, Hk, D, Rt, layout, norm, affine, bias, fused, index, batches = case
    x = inputs(B, L, H, Hk, D, Rt, fused, index, batches, affine, bias)
    kw = dict(index=x["index"], norm=norm, layout=layout, **{n: x[n] for n in ("q_weight", "k_weight", "q_bias", "k_bias")})
    q, k, tq, tk = aj.qk_rotary_jvp(x["q"], x["k"], x["table"], **kw, tq=x["tq"], tk=x["tk"])
    q2, k2, none, none2 = aj.qk_rotary_jvp(x["q"], x["k"], x["table"], **kw)
    assert none is None and none2 is None and torch.equal(q, q2) and (k is None) == (Hk == 0)
    assert Hk == 0 or torch.equal(k, k2)
    grads = aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw)
    again = aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw)
    for a, b in zip(grads, again):
        assert (a is None and b is None) or torch.equal(a, b)
    cs = R.rows_of(x["table"], x["index"], B, L)
    for n, y, ty, dx in (("q", q, tq, grads.q), ("k", k, tk, grads.k)):
        if x[n] is None:
            assert y is None and ty is None and dx is None
            continue
        assert y.is_contiguous() and dx.is_contiguous() and y.shape == x[n].shape
        one, zero = torch.ones(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
        w = one if x[n + "_weight"] is None else x[n + "_weight"].double()
        b = zero if x[n + "_bias"] is None else x[n + "_bias"].double()
        x64 = x[n].double()
        want, twant = torch.func.jvp(lambda v: R.head(v, cs, w, b, norm, layout), (x64,), (x["t" + n].double(),))
        # sizes of the terms: of u, and of the normalisation's derivative before its parts cancel
        c = x64 - x64.mean(-1, keepdim=True) if norm == "layer" else x64
        r = torch.ones_like(c[..., :1]) if norm is None else 1 / torch.sqrt(c.square().mean(-1, keepdim=True) + R.EPS)
        big = x64.abs().amax(-1, keepdim=True) * r
        wm, bm = w.abs().amax(), b.abs().amax()
        close(n, y, want, big * wm + bm)
        t64 = x["t" + n].double().abs().amax(-1, keepdim=True)
        close("t" + n, ty, twant, r * t64 * wm * (1 + big * (c * r).abs().amax(-1, keepdim=True)))
        dy = x["d" + n].double()
        args = [t.clone().requires_grad_() for t in (x64, w, b)]
        dxw, dww, dbw = torch.autograd.grad(R.head(args[0], cs, args[1], args[2], norm, layout), args, dy)
        dmax = 2 * dy.abs().amax(-1, keepdim=True)
        close("d" + n, dx, dxw, r * dmax * wm * (1 + big * (c * r).abs().amax(-1, keepdim=True)))
        du = R.turn(dy, cs * torch.tensor([1.0, -1.0], device="cuda", dtype=torch.float64), layout)
        # (a term's own rounding: du and n are each some ten operations old)
        for m, got, wanted, size in (("weight", getattr(grads, n + "_weight"), dww, (dmax * big).sum((0, 1, 2))),
                                     ("bias", getattr(grads, n + "_bias"), dbw, dmax.expand_as(dy).sum((0, 1, 2)))):
            assert (got is None) == (x[f"{n}_{m}"] is None)
            if got is not None:
                assert ((got.double() - wanted).abs() <= 2.0 ** -24 * 340 * size).all(), m
        assert du.shape == dy.shape
    torch.cuda.synchronize()
    assert aj.attn_jvp_device_status() == 0


@pytest.mark.parametrize("norm,layout", list(itertools.product(["rms", "layer", None], ["interleaved", "half"])))
def test_gradients_against_differences(aj, norm, layout):
    """Along directions of its own, the definition's differences (64 bits) agree with the kernel's gradients."""
    B, L, H, Hk, D, Rt = 2, 37, 3, 2, 64, 48
    x = inputs(B, L, H, Hk, D, Rt, False, 0, False, True, True, seed=5)
    kw = dict(norm=norm, layout=layout, **{n: x[n] for n in ("q_weight", "k_weight", "q_bias", "k_bias")})
    g = aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw)
    cs = R.rows_of(x["table"], None, B, L)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for n in "qk":
        args = [x[n].double(), x[n + "_weight"].double(), x[n + "_bias"].double()]
        for i, grad in enumerate((getattr(g, n), getattr(g, n + "_weight"), getattr(g, n + "_bias"))):
            way = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
            h = 1e-5
            f = lambda s: (R.head(*[a + (s * way if j == i else 0) for j, a in enumerate(args[:1])], cs, args[1] + (s * way if i == 1 else 0),
                                  args[2] + (s * way if i == 2 else 0), norm, layout) * x["d" + n].double()).sum()
            want = (f(h) - f(-h)) / (2 * h)
            got = (grad.double() * way).sum()
            # one rounding to bf16 per element (2^-8 of it, random signs: six deviations of the sum), fp32 sums, differences good to 1e-6
            size = (grad.double() * way).square().sum().sqrt()
            assert (got - want).abs() <= 6 * 2.0 ** -8 * size + 1e-6 * (1 + want.abs() + (grad.double() * way).abs().sum()), (n, i)


def test_rows_do_not_touch_each_other(aj):
    """A NaN or infinity stays in its row; an index outside the table reads its nearest row."""
    x = inputs(2, 50, 5, 2, 128, 64, False, 1, False, True, False)
    kw = dict(norm="rms", q_weight=x["q_weight"], k_weight=x["k_weight"])
    clean = aj.qk_rotary_jvp(x["q"], x["k"], x["table"], index=x["index"], **kw)
    q = x["q"].clone()
    q[1, 7, 3, 100], q[0, 49, 4, 0] = float("nan"), float("inf")
    got = aj.qk_rotary_jvp(q, x["k"], x["table"], index=x["index"], **kw)
    same = (got[0] == clean[0]).all(-1)
    assert not same[1, 7, 3] and not same[0, 49, 4] and same.sum() == same.numel() - 2 and torch.equal(got[1], clean[1])
    rows = x["table"].shape[0]
    wild = x["index"].clone()
    wild[3], wild[9] = -5, rows + 1000
    tame = wild.clamp(0, rows - 1)
    for a, b in zip(aj.qk_rotary_jvp(x["q"], x["k"], x["table"], index=wild, **kw)[:2],
                    aj.qk_rotary_jvp(x["q"], x["k"], x["table"], index=tame, **kw)[:2]):
        assert torch.equal(a, b)


def test_heads_before_tokens(aj):
    """Tensors that lie as [B][H][L][D]."""
    x = inputs(2, 77, 5, 3, 64, 64, False, 0, False, True, False)
    kw = dict(norm="rms", layout="half", q_weight=x["q_weight"], k_weight=x["k_weight"])
    other = {n: x[n].transpose(1, 2).contiguous().transpose(1, 2) for n in ("q", "k", "tq", "tk")}
    assert not other["q"].is_contiguous()
    for a, b in zip(aj.qk_rotary_jvp(x["q"], x["k"], x["table"], **kw, tq=x["tq"], tk=x["tk"]),
                    aj.qk_rotary_jvp(other["q"], other["k"], x["table"], **kw, tq=other["tq"], tk=other["tk"])):
        assert torch.equal(a, b)
    for a, b in zip(aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw),
                    aj.qk_rotary_backward(x["dq"], x["dk"], other["q"], other["k"], x["table"], **kw)):
        assert (a is None and b is None) or torch.equal(a, b)


def test_far_strides(aj):
    """Offsets beyond 2^31 elements."""
    B, L, H, D = 2, 3, 2, 64
    far = (1 << 31) + 64
    buffer = torch.empty(far + L * H * D, dtype=torch.bfloat16, device="cuda")
    q = buffer.as_strided((B, L, H, D), (far, H * D, D, 1))
    near = torch.randn(B, L, H, D, device="cuda").bfloat16()
    q.copy_(near)
    t = aj.rotary_table(torch.arange(L, device="cuda"), D)
    assert torch.equal(aj.qk_rotary_jvp(q, None, t, norm="rms")[0], aj.qk_rotary_jvp(near, None, t, norm="rms")[0])


def test_refusals(aj):
    x = inputs(2, 20, 4, 2, 64, 32, False, 0, False, True, True)
    ok = dict(q=x["q"], k=x["k"], table=x["table"])
    bad = [dict(q=x["q"].float()), dict(q=x["q"].cpu()), dict(q=x["q"][0]), dict(k=x["k"][:1]), dict(k=x["k"][:, :, :, :32]),
           dict(table=x["table"][:19]), dict(table=x["table"].double()), dict(table=x["table"][..., :1]), dict(table=x["table"][None].expand(3, -1, -1, -1).contiguous()),
           dict(index=torch.zeros(21, dtype=torch.int32, device="cuda")), dict(index=torch.zeros(20, device="cuda")), dict(norm="batch"), dict(layout="thirds"),
           dict(q_weight=x["q_weight"][:32]), dict(q_weight=x["q_weight"].half()), dict(k=None, k_weight=x["k_weight"]), dict(tk=x["tk"]), dict(tq=x["tq"]),
           dict(q=x["q"].transpose(2, 3).contiguous().transpose(2, 3)), dict(q=torch.empty(2, 20, 4 * 64 + 4, device="cuda").bfloat16()[..., :256].view(2, 20, 4, 64)),
           dict(eps=float("nan")), dict(table=x["table"][:, :3].contiguous()), dict(q=torch.zeros(2, 20, 4, 96, device="cuda").bfloat16(), k=None), dict(q=x["q"][:, :0])]
    for b in bad:
        with pytest.raises((ValueError, aj.AttnJvpError)):
            aj.qk_rotary_jvp(**{**ok, **b})
    d = dict(dq_new=x["dq"], dk_new=x["dk"], **ok)
    for b in (dict(dk_new=None), dict(dq_new=None), dict(dq_new=x["dq"].transpose(1, 2)), dict(k=None), dict(q_weight=x["q_weight"], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, aj.AttnJvpError)):
            aj.qk_rotary_backward(**{**d, **b})


def test_own_workspace_stream_and_capture(aj):
    x = inputs(1, 300, 6, 3, 128, 128, True, 0, False, True, False)
    kw = dict(norm="rms", q_weight=x["q_weight"], k_weight=x["k_weight"])
    need = aj.attn_jvp_qk_rotary_bwd_workspace_bytes(1, 300, 6, 3, 128)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    call = lambda w=None: (*aj.qk_rotary_jvp(x["q"], x["k"], x["table"], **kw, tq=x["tq"], tk=x["tk"]),
                           *aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw, workspace=w)[:4])
    want = call()
    for a, b in zip(call(ws[:need]), want):
        assert torch.equal(a, b)
    assert (ws[need:] == 255).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_layer(aj):
    """Autograd, JVP pairs, no keys, and that the layer's own gradients have none."""
    x = inputs(2, 40, 4, 2, 64, 64, True, 0, False, False, False)
    layer = aj.QKRotaryJVP(64, bias=True).cuda()
    with torch.no_grad():
        for p in layer.parameters():
            p.add_(torch.randn_like(p) * 0.2)
    q, k = (x[n].clone().requires_grad_() for n in "qk")
    y = layer(q, k, x["table"])
    grads = torch.autograd.grad(y, (q, k, *layer.parameters()), (x["dq"], x["dk"]))
    want = aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], norm="rms", q_weight=layer.q_weight.detach(), k_weight=layer.k_weight.detach(),
                                 q_bias=layer.q_bias.detach(), k_bias=layer.k_bias.detach())
    for a, b in zip(grads, want):
        assert torch.equal(a, b)
    (q2, tq2), (k2, tk2) = layer((x["q"], x["tq"]), (x["k"], x["tk"]), x["table"], withT=True)
    assert torch.equal(q2, y[0]) and torch.equal(k2, y[1]) and not q2.requires_grad and tq2.shape == q2.shape and tk2.shape == k2.shape
    alone = aj.QKRotaryJVP(64, affine=False)
    assert torch.equal(alone(x["q"], None, x["table"]), aj.qk_rotary_jvp(x["q"], None, x["table"], norm="rms")[0])
    assert alone((x["q"], x["tq"]), None, x["table"], withT=True)[1].shape == x["q"].shape
    (only,) = torch.autograd.grad(layer(q, k, x["table"])[0], q, x["dq"])
    assert torch.equal(only, want.q)
    (g,) = torch.autograd.grad(layer(q, k, x["table"])[0].float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()
    with pytest.raises(ValueError):
        layer((x["q"], x["tq"]), x["k"], x["table"], withT=True)
