"""Fused gate + residual + norm + modulation (forward, tangents, gradients) against its 64-bit statement.

Tolerances.  Inputs are exact in fp64.  The kernel's arithmetic is fp32: a row's sums run over 8 channels in a thread,
5 + 5 shuffle levels and at most 32 warps, so they carry at most about 20 roundings of 2^-24 relative to the sum of
magnitudes, and a value then goes through fewer than 20 further operations: 40 * 2^-24 = 2.4e-6 of the largest magnitude
that enters it.  ARITH = 1e-5 of the output's largest value covers it four times over.  On top, half a step of the
stored type: 2^-8 of the value for bf16, 2^-24 for fp32.  Column sums over tokens add one rounding per token and CTA:
(tokens + 64) * 2^-24 of the sum of magnitudes.  Their terms are products a b of two such values of a row (dx hn, dy n),
each off by ARITH of its row's largest, whatever its own size (dx is a difference that may cancel at one channel):
|a' b' - a b| <= ARITH (max|a| |b| + |a| max|b|) + ARITH^2 max|a| max|b|, summed over the tokens.
"""
import pytest
import torch

from tests import adaln_ref

pytestmark = pytest.mark.gpu
ARITH = 1e-5
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def close(name, got, ref, extra=None):
    assert got.shape == ref.shape, name
    g = got.double()
    assert torch.isfinite(g).all(), f"{name}: non-finite"
    tol = HALF[got.dtype] * ref.abs() + (ARITH * ref.abs().max() if extra is None else extra)
    bad = (g - ref).abs() - tol
    assert bad.max() <= 0, f"{name}: off by {(g - ref).abs().max():.3g}, {bad.max():.3g} over"


def make(B, L, C, xt, has_h=True, mods=("gate", "scale", "shift"), weights=True, seed=0, layout="sliced"):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * C + L)
    rn = lambda *s, sigma=1.0: torch.randn(*s, generator=g, device="cuda") * sigma  # noqa: E731
    a = dict(x=rn(B, L, C).to(xt), h=rn(B, L, C).bfloat16() if has_h else None)
    block = rn(B, 6, C + 1, sigma=0.5)[:, :, 1:]        # odd row stride: rows are 4-byte aligned only
    if layout == "shared":
        block = block[:1].expand(B, 6, C)
    if layout == "aligned":
        block = rn(B, 6, C, sigma=0.5)
    for i, n in enumerate(("gate", "scale", "shift")):
        a[n] = block[:, i] if n in mods and (n != "gate" or has_h) else None
    a["weight"] = 1 + rn(C, sigma=0.2) if weights else None
    a["post_weight"] = 1 + rn(C, sigma=0.2) if weights and has_h else None
    t = dict(tx=rn(B, L, C, sigma=0.5).to(xt), th=rn(B, L, C, sigma=0.5).bfloat16() if has_h else None)
    for i, n in enumerate(("gate", "scale", "shift")):
        t["t" + n] = block[:, 3 + i] if a[n] is not None else None
    d = dict(dx_new=rn(B, L, C).to(xt), dy=rn(B, L, C).bfloat16())
    return a, t, d


def f64(t):
    return None if t is None else t.double()


KEYS = ("x", "h", "gate", "scale", "shift", "weight", "post_weight")


def reference(a, norm, post, eps, t=None, d=None):
    vals = [f64(a[k]) for k in KEYS]
    at = [i for i, v in enumerate(vals) if v is not None]

    def f(*some):
        full = list(vals)
        for i, v in zip(at, some):
            full[i] = v
        out = adaln_ref.step(*full, norm, post, eps)
        return out[:1] if out[1] is None else out

    prim = tuple(vals[i] for i in at)
    if t is not None:
        tan = tuple(torch.zeros_like(vals[i]) if t.get("t" + KEYS[i]) is None else t["t" + KEYS[i]].double() for i in at)
        return torch.func.jvp(f, prim, tan)
    if d is None:
        return f(*prim)
    prim = [p.clone().requires_grad_() for p in prim]
    out = f(*prim)
    cot = [None if c is None else c.double() for c in (d["dx_new"], d["dy"])][:len(out)]
    pairs = [(o, c) for o, c in zip(out, cot) if c is not None]
    grads = torch.autograd.grad([o for o, _ in pairs], prim, [c for _, c in pairs], allow_unused=True)
    return {KEYS[i]: (torch.zeros_like(p) if g is None else g) for i, p, g in zip(at, prim, grads)}


SHAPES = [(1, 1, 8), (2, 3, 64), (1, 130, 264), (3, 257, 1536), (1, 37, 2048), (2, 301, 5120), (1, 9, 5128), (2, 5, 8192)]


@pytest.mark.parametrize("B,L,C", SHAPES)
@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm,post", [("layer", None), ("rms", "layer"), ("layer", "rms")])
def test_forward_and_tangents(aj, B, L, C, xt, norm, post):
    a, t, _ = make(B, L, C, xt)
    x, y, tx, ty = aj.adaln_jvp(**a, norm=norm, post_norm=post, eps=1e-6, **t)
    (rx, ry), (rtx, rty) = reference(a, norm, post, 1e-6, t=t)
    assert x.dtype == tx.dtype == xt and y.dtype == ty.dtype == torch.bfloat16
    for n, g, r in (("x'", x, rx), ("y", y, ry), ("tx'", tx, rtx), ("ty", ty, rty)):
        close(n, g, r)
    x2, y2, none1, none2 = aj.adaln_jvp(**a, norm=norm, post_norm=post, eps=1e-6)
    assert none1 is None and none2 is None
    close("x' without tangents", x2, rx)
    close("y without tangents", y2, ry)


def grad_checks(aj, a, d, norm, post, g):
    ref = reference(a, norm, post, 1e-6, d=d)
    B, L, C = a["x"].shape
    # column sums: magnitudes of what is summed
    vals = {k: f64(v) for k, v in a.items()}
    xn = adaln_ref.step(*[vals[k] for k in KEYS], None, post, 1e-6)[0]
    tol = {}

    def column(a, b, factor, dims):
        """Tolerance of sum over `dims` of a b, scaled by |factor| ([B][1][C] or [C])."""
        top_a, top_b = a.abs().amax(-1, keepdim=True), b.abs().amax(-1, keepdim=True)
        each = (L + 64) * 2.0 ** -24 * (a * b).abs() + ARITH * (top_a * b.abs() + a.abs() * top_b) + ARITH ** 2 * top_a * top_b
        return (each * factor).sum(dims)

    one = torch.ones(C, dtype=torch.float64, device="cuda")
    if norm is not None and d["dy"] is not None:
        n, dy = adaln_ref.normed(xn, norm, 1e-6), d["dy"].double()
        w = one if vals["weight"] is None else vals["weight"].abs()
        s = one if vals["scale"] is None else (1 + vals["scale"]).abs()[:, None]
        tol = dict(scale=column(dy, n, w, 1), shift=(L + 64) * 2.0 ** -24 * dy.abs().sum(1), weight=column(dy, n, s, (0, 1)))
    if a["h"] is not None:
        hn = adaln_ref.normed(vals["h"], post, 1e-6)
        wp = one if vals["post_weight"] is None else vals["post_weight"].abs()
        gt = one if vals["gate"] is None else vals["gate"].abs()[:, None]
        tol.update(gate=column(ref["x"], hn, wp, 1), post_weight=column(ref["x"], hn, gt, (0, 1)))
    for k in KEYS:
        got = getattr(g, k)
        assert (got is None) == (a[k] is None), k
        if got is None:
            continue
        if k in ("x", "h"):
            close("d" + k, got, ref[k])
        else:
            close("d" + k, got, ref[k], extra=tol.get(k, 0.0) + 1e-30)


@pytest.mark.parametrize("B,L,C", SHAPES)
@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm,post", [("layer", None), ("rms", "layer"), ("layer", "rms")])
def test_gradients(aj, B, L, C, xt, norm, post):
    a, _, d = make(B, L, C, xt)
    g = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm=norm, post_norm=post, eps=1e-6)
    grad_checks(aj, a, d, norm, post, g)


@pytest.mark.parametrize("B,L,C,xt", [(1, 7301, 1536, torch.bfloat16), (2, 9001, 520, torch.bfloat16), (1, 57001, 64, torch.bfloat16),
                                      (1, 7200, 2048, torch.bfloat16), (1, 150, 5120, torch.bfloat16), (3, 50, 2056, torch.float32),
                                      (1, 1, 4096, torch.float32)])
@pytest.mark.parametrize("norm,has_h", [("layer", True), ("rms", True), ("layer", False)])
def test_long_runs_without_a_post_norm(aj, B, L, C, xt, norm, has_h):
    """The rows of a CTA overlap here (a row's sums are formed while the row before is finished), in every combination."""
    a, t, d = make(B, L, C, xt, has_h=has_h)
    x, y, tx, ty = aj.adaln_jvp(**a, norm=norm, eps=1e-6, **t)
    (rx, ry), (rtx, rty) = reference(a, norm, None, 1e-6, t=t)
    for n, g, r in (("x'", x, rx), ("y", y, ry), ("tx'", tx, rtx), ("ty", ty, rty)):
        close(n, g, r)
    for dx_new, dy in ((d["dx_new"], d["dy"]), (None, d["dy"]), (d["dx_new"], None)):
        g = aj.adaln_backward(dx_new, dy, **a, norm=norm, eps=1e-6)
        grad_checks(aj, a, dict(dx_new=dx_new, dy=dy), norm, None, g)
    for u, v in zip(aj.adaln_backward(d["dx_new"], d["dy"], **a, norm=norm), aj.adaln_backward(d["dx_new"], d["dy"], **a, norm=norm)):
        assert u is v or torch.equal(u, v)


@pytest.mark.parametrize("mods", [(), ("scale",), ("gate", "shift"), ("shift",)])
@pytest.mark.parametrize("norm,post,has_h", [("layer", None, False), ("rms", None, False), (None, "rms", True), (None, None, True),
                                             ("layer", None, True)])
def test_optional_parts(aj, mods, norm, post, has_h):
    mods = tuple(m for m in mods if (norm is not None or m == "gate") and (has_h or m != "gate"))
    a, t, d = make(2, 33, 1544, torch.float32, has_h=has_h, mods=mods, weights=False)
    x, y, tx, ty = aj.adaln_jvp(**a, norm=norm, post_norm=post, eps=1e-6, **t)
    out, tan = reference(a, norm, post, 1e-6, t=t)
    close("x'", x, out[0])
    close("tx'", tx, tan[0])
    if norm is None:
        assert y is None and ty is None
    else:
        close("y", y, out[1])
        close("ty", ty, tan[1])
    if not has_h:
        assert x is a["x"] and tx is t["tx"]
    for dx_new, dy in ((d["dx_new"], d["dy"]), (None, d["dy"]), (d["dx_new"], None)):
        if norm is None:
            dy = None
        if dx_new is None and dy is None:
            continue
        g = aj.adaln_backward(dx_new, dy, **a, norm=norm, post_norm=post, eps=1e-6)
        grad_checks(aj, a, dict(dx_new=dx_new, dy=dy), norm, post, g)


@pytest.mark.parametrize("layout", ["aligned", "shared"])
def test_modulation_layouts(aj, layout):
    """Aligned rows take 16-byte loads, rows shared by every batch have stride 0; gradients come per sample."""
    a, t, d = make(3, 65, 512, torch.bfloat16, layout=layout)
    x, y, tx, ty = aj.adaln_jvp(**a, norm="layer", eps=1e-6, **t)
    (rx, ry), (rtx, rty) = reference(a, "layer", None, 1e-6, t=t)
    for n, g, r in (("x'", x, rx), ("y", y, ry), ("tx'", tx, rtx), ("ty", ty, rty)):
        close(n, g, r)
    grad_checks(aj, a, d, "layer", None, aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="layer", eps=1e-6))


def test_long_sequence_and_repeatability(aj):
    """Every CTA walks many rows; two calls give the same bits (no atomics)."""
    a, _, d = make(1, 5001, 1536, torch.bfloat16)
    g = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="layer", eps=1e-6)
    grad_checks(aj, a, d, "layer", None, g)
    g2 = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="layer", eps=1e-6)
    for u, v in zip(g, g2):
        assert u is None or torch.equal(u, v)


def test_many_short_batches(aj):
    a, t, d = make(700, 2, 72, torch.float32)
    x, y, _, _ = aj.adaln_jvp(**a, norm="layer", eps=1e-6)
    rx, ry = reference(a, "layer", None, 1e-6)
    close("x'", x, rx)
    close("y", y, ry)
    grad_checks(aj, a, d, "layer", None, aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="layer", eps=1e-6))


@pytest.mark.parametrize("C", [64, 1536, 5120])
def test_rows_whose_mean_is_far_from_zero(aj, C):
    """x = 4096 + noise is exact to 2^-12 in fp32; its variance must not drown in the squared mean.  The mean carries at
    most 20 roundings of 2^-24 * 4096 (5e-3 after 20; measured against deviation 1 the shift of all n alike), which is
    what the tolerance allows."""
    g = torch.Generator(device="cuda").manual_seed(C)
    x = 4096 + torch.randn(2, 7, C, generator=g, device="cuda")
    _, y, _, _ = aj.adaln_jvp(x, norm="layer", eps=1e-6)
    ref = adaln_ref.normed(x.double(), "layer", 1e-6)
    assert (y.double() - ref).abs().max() <= 2.0 ** -8 * ref.abs().max() + 20 * 4096 * 2.0 ** -24
    _, y, _, ty = aj.adaln_jvp(x, norm="layer", eps=1e-6, tx=torch.zeros_like(x))
    assert (y.double() - ref).abs().max() <= 2.0 ** -8 * ref.abs().max() + 20 * 4096 * 2.0 ** -24 and not ty.any()


def test_constant_and_zero_rows(aj):
    """Deviation 0: n is 0 (eps keeps it finite), so y is the shift alone."""
    x = torch.zeros(1, 3, 1536, device="cuda")
    x[:, 1] = 2.0
    shift = torch.randn(1, 1536, device="cuda")
    _, y, _, _ = aj.adaln_jvp(x, shift=shift, norm="layer", eps=1e-6)
    assert torch.equal(y, shift.bfloat16().expand(1, 3, 1536))


def test_gradient_against_differences(aj):
    """<gradient, direction> = central difference of the 64-bit step along the direction (fp32 x, so that the kernel's dx
    is not rounded to bf16; dh is: its share of the product gets half a bf16 step per element)."""
    a, _, d = make(2, 5, 256, torch.float32, seed=3)
    g = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="layer", post_norm="rms", eps=1e-4)
    gen = torch.Generator(device="cuda").manual_seed(11)
    vals = {k: a[k].double() for k in KEYS}
    dirs = {k: torch.randn(v.shape, generator=gen, device="cuda", dtype=torch.float64) for k, v in vals.items()}

    def loss(e):
        xn, y = adaln_ref.step(*[vals[k] + e * dirs[k] for k in KEYS], "layer", "rms", 1e-4)
        return (xn * d["dx_new"].double()).sum() + (y * d["dy"].double()).sum()

    e = 1e-5
    want = (loss(e) - loss(-e)) / (2 * e)
    terms = {k: getattr(g, k).double() * dirs[k] for k in KEYS}
    got = sum(v.sum() for v in terms.values())
    tol = sum(v.abs().sum() for v in terms.values()) * ARITH + terms["h"].abs().sum() * 2.0 ** -8 + 1e-4
    assert abs(got - want) <= tol


def test_streams_graphs_and_workspace(aj):
    """Captured and replayed on new inputs, on a side stream, with a caller's workspace."""
    a, t, d = make(2, 100, 640, torch.bfloat16)
    b, tb, db = make(2, 100, 640, torch.bfloat16, seed=5)
    ws = torch.empty(aj.attn_jvp_adaln_bwd_workspace_bytes(2, 100, 640), dtype=torch.uint8, device="cuda")
    want_f = aj.adaln_jvp(**b, norm="rms", **tb)
    want_g = aj.adaln_backward(db["dx_new"], db["dy"], **b, norm="rms")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            f = aj.adaln_jvp(**a, norm="rms", **t)
            g = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="rms", workspace=ws)
        for src, dst in ((b, a), (tb, t), (db, d)):
            for k in src:
                if k in ("gate", "scale", "shift", "tgate", "tscale", "tshift"):
                    dst[k].copy_(src[k])
                else:
                    dst[k].copy_(src[k])
        graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(list(f) + list(g), list(want_f) + list(want_g)):
        assert torch.equal(u, v)


def test_rows_behind_the_last_are_left_alone(aj):
    """Outputs are written for B * L rows and no further."""
    a, t, d = make(1, 3, 264, torch.bfloat16, weights=False)
    n = 3 * 264
    buf = [torch.full((n + 512,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    args = aj.AdaLNArgs(B=1, L=3, C=264, norm=1, eps=1e-6)
    for k, v in {**a, **t}.items():
        if v is not None:
            setattr(args, k, v.data_ptr())
    assert aj.attn_jvp_adaln_fwd(args, *buf, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for b in buf:
        assert (b[n:] == 7.0).all() and (b[:n] != 7.0).any()


def test_outputs_between_sectors(aj):
    """fp32 tensors 16 bytes off a 32-byte boundary, as the boundary allows: the same bits as the aligned ones."""
    a, t, d = make(2, 21, 1288, torch.float32)
    n = a["x"].numel()
    want = aj.adaln_jvp(**a, norm="rms", post_norm="layer", **t)
    want_g = aj.adaln_backward(d["dx_new"], d["dy"], **a, norm="rms", post_norm="layer")

    def off(v=None):
        buf = torch.full((n + 8,), 7.0, device="cuda")
        assert buf.data_ptr() % 32 == 0
        if v is not None:
            buf[4:n + 4] = v.reshape(-1)
        return buf

    ins = dict(x=off(a["x"]), tx=off(t["tx"]))
    args = aj.AdaLNArgs(B=2, L=21, C=1288, norm=2, post_norm=1, eps=1e-6, x_dtype=1)
    for k, v in {**a, **t}.items():
        setattr(args, k, ins[k][4:].data_ptr() if k in ins else v.data_ptr())
        if v.dim() == 2:
            setattr(args, k + "_stride", v.stride(0))
    xn, txn, dx, dxn = off(), off(), off(), off(d["dx_new"])
    y, ty, dh = (torch.empty_like(a["h"]) for _ in range(3))
    st = torch.cuda.current_stream().cuda_stream
    assert aj.attn_jvp_adaln_fwd(args, xn[4:], y, txn[4:], ty, st) == 0
    g = [torch.empty(2, 1288, device="cuda") for _ in range(3)] + [torch.empty(1288, device="cuda") for _ in range(2)]
    ws = torch.empty(aj.attn_jvp_adaln_bwd_workspace_bytes(2, 21, 1288), dtype=torch.uint8, device="cuda")
    assert aj.attn_jvp_adaln_bwd(args, dxn[4:], d["dy"], dx[4:], dh, *g, ws, ws.numel(), st) == 0
    torch.cuda.synchronize()
    for got, ref in zip((xn, txn, dx), (want[0], want[2], want_g.x)):
        assert torch.equal(got[4:n + 4], ref.reshape(-1)) and (got[:4] == 7.0).all() and (got[n + 4:] == 7.0).all()
    for got, ref in zip([y, ty, dh] + g, [want[1], want[3], want_g.h, want_g.gate, want_g.scale, want_g.shift, want_g.weight, want_g.post_weight]):
        assert torch.equal(got, ref)


def test_workspace_must_be_large_enough(aj):
    a, _, d = make(1, 40, 64, torch.bfloat16)
    need = aj.attn_jvp_adaln_bwd_workspace_bytes(1, 40, 64)
    with pytest.raises(aj.AttnJvpError) as e:
        aj.adaln_backward(d["dx_new"], d["dy"], **a, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 12
