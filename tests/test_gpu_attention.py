"""Dense attention with a causal mask, key lengths, shared key heads and strided inputs: forward, tangents and gradients against the 64-bit
statement in tests/attention_ref.py (which says where the tolerances come from)."""
import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def inputs(B, H, Hk, Lq, Lk, D, fused=False, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + Lq + 3 * Lk + 7 * H)
    rn = lambda *s, f=1.0: (torch.randn(*s, generator=g, device="cuda") * f).bfloat16()
    x = dict(q=rn(B, Lq, H, D), k=rn(B, Lk, Hk, D), v=rn(B, Lk, Hk, D), tq=rn(B, Lq, H, D, f=0.7), tk=rn(B, Lk, Hk, D, f=0.7), tv=rn(B, Lk, Hk, D, f=0.7),
             d_o=rn(B, Lq, H, D))
    if fused:
        y = rn(B, Lk, H + 2 * Hk, D)
        x.update(q=y[:, :Lq, :H], k=y[:, :, H:H + Hk], v=y[:, :, H + Hk:])
    return x


def no_timeout(aj):
    torch.cuda.synchronize()
    st = aj.attn_jvp_device_status()
    assert st == 0, (aj.attn_jvp_strerror(st), aj.attn_jvp.attn_jvp_debug_timeout_info())


def run_all(aj, x, causal=False, lengths=None, scale=None, tangents=True):
    s = x["q"].shape[-1] ** -0.5 if scale is None else scale
    kl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(scale=scale, causal=causal, k_lengths=kl)
    o, none, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, **kw)
    no_timeout(aj)
    assert none is None
    ref = R.attention(x["q"], x["k"], x["v"], s, causal, lengths, x["tq"], x["tk"], x["tv"], x["d_o"])
    R.check("o", o, ref["o"])
    R.check("lse", lse, ref["lse"])
    dq, dk, dv = aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, **kw)
    no_timeout(aj)
    for n, g in dict(dq=dq, dk=dk, dv=dv).items():
        assert g.is_contiguous()
        R.check(n, g, ref[n])
    if tangents:
        got = aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], x["tk"], x["tv"], return_mu=True, **kw)
        no_timeout(aj)
        for n, g in zip(("o", "to", "lse", "mu"), got):
            R.check(n + " (tangents)", g, ref[n.split()[0]])
        free = R.attention(x["q"], x["k"], x["v"], s, causal, lengths, x["tq"])
        got = aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], return_mu=True, **kw)
        no_timeout(aj)
        for n, g in zip(("o", "to", "lse", "mu"), got):
            R.check(n + " (constant context)", g, free[n])
    return o, lse, dq, dk, dv


SIZES = [(1, 1), (1, 333), (64, 65), (128, 128), (129, 64), (200, 333), (333, 192), (517, 1000), (1000, 257), (383, 385)]


@pytest.mark.parametrize("Lq,Lk", SIZES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_sizes(aj, Lq, Lk, D, causal):
    """Own and shared heads, every length from none to all; under the causal mask with Lq > Lk the first rows see nothing."""
    run_all(aj, inputs(2, 3, 3, Lq, Lk, D), causal, tangents=causal)
    run_all(aj, inputs(3, 4, 2, Lq, Lk, D, seed=5), causal, [Lk, 0, max(1, Lk // 2)])
    run_all(aj, inputs(2, 6, 1, Lq, Lk, D, seed=6), causal, [max(1, Lk - 1), Lk + 7], tangents=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths", [[1, 2, 127], [128, 129, 255], [256, 300, 64], [0, 0, 0], [-4, 1000, 65]])
def test_lengths(aj, D, lengths):
    for causal in (False, True):
        run_all(aj, inputs(3, 2, 1, 300, 300, D), causal, lengths)


@pytest.mark.parametrize("B", [31, 32, 33, 40])
@pytest.mark.parametrize("causal", [False, True])
def test_many_batches_some_without_keys(aj, B, causal):
    lengths = [0 if b % 3 == 1 else 1 + (37 * b) % 200 for b in range(B)]
    run_all(aj, inputs(B, 2, 1, 150, 200, 64), causal, lengths)
    run_all(aj, inputs(B, 1, 1, 150, 200, 128), causal, [0] * (B - 1) + [130], tangents=False)


@pytest.mark.parametrize("D", [64, 128])
def test_more_items_than_multiprocessors(aj, D):
    for causal in (False, True):
        run_all(aj, inputs(2, 14, 7, 1100, 1100, D), causal, [1100, 900])
        run_all(aj, inputs(2, 14, 14, 1500, 1100, D), causal)


@pytest.mark.parametrize("D", [64, 128])
def test_few_blocks_and_a_long_other_side(aj, D):
    """Items cut into parts whose sums are joined: keys few, then queries few; parts that a mask leaves empty among them."""
    run_all(aj, inputs(1, 2, 1, 5000, 200, D), lengths=[150], tangents=False)
    run_all(aj, inputs(1, 2, 2, 200, 5000, D), tangents=False)
    run_all(aj, inputs(2, 2, 2, 100, 5000, D), lengths=[5000, 130], tangents=False)
    run_all(aj, inputs(1, 2, 2, 5000, 300, D), causal=True, tangents=False)
    run_all(aj, inputs(1, 1, 1, 3000, 3000, D), causal=True, tangents=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.11, 0.3])
def test_scales(aj, D, scale):
    run_all(aj, inputs(2, 2, 1, 300, 450, D), True, [450, 200], scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_slices_of_one_projection(aj, D):
    x = inputs(2, 4, 2, 300, 300, D, fused=True)
    assert not x["q"].is_contiguous()
    got = run_all(aj, x, True, [300, 170])
    y = {n: t.contiguous() for n, t in x.items()}
    for a, b in zip(got, run_all(aj, y, True, [300, 170], tangents=False)):
        assert torch.equal(a, b)
    run_all(aj, x)


@pytest.mark.parametrize("D", [64, 128])
def test_heads_before_tokens_and_far_batches(aj, D):
    """Tensors that lie as [B][H][L][D], and batches more than 2^31 elements apart."""
    B, H, Hk, L, lengths = 2, 4, 2, 200, [200, 130]
    x = inputs(B, H, Hk, L, L, D)
    want = run_all(aj, x, True, lengths, tangents=False)
    y = dict(x, **{n: x[n].transpose(1, 2).contiguous().transpose(1, 2) for n in "qkv"})
    assert not y["q"].is_contiguous()
    for a, b in zip(run_all(aj, y, True, lengths), want):
        assert torch.equal(a, b)
    far = (1 << 31) + 64
    buffer = torch.empty(far + L * (H + 2 * Hk) * D, dtype=torch.bfloat16, device="cuda")
    at = 0
    for n in "qkv":
        h = x[n].shape[2]
        y[n] = buffer[at:].as_strided(x[n].shape, (far, h * D, D, 1))
        y[n].copy_(x[n])
        at += L * h * D
    for a, b in zip(run_all(aj, y, True, lengths, tangents=False), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_padding_may_hold_anything(aj, D, causal):
    """NaN and infinities behind a batch's keys reach nothing: results are those of zeros there, bit for bit."""
    lengths = [130, 0, 256]
    outs = []
    for fill in (0.0, float("nan"), float("inf")):
        x = inputs(3, 4, 2, 384, 384, D)
        for b, n in enumerate(lengths):
            for t in ("k", "v", "tk", "tv"):
                x[t][b, n:] = fill
        kl = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        kw = dict(causal=causal, k_lengths=kl)
        o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, **kw)
        outs.append((o, lse, *aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, **kw),
                     *aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], x["tk"], x["tv"], return_mu=True, **kw),
                     *aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], return_mu=True, **kw)))
        no_timeout(aj)
    for i, (a, b, c) in enumerate(zip(*outs)):
        assert torch.equal(a, b) and torch.equal(a, c), i
        assert (a[1] == 0).all() or (a[1] == -float("inf")).all()          # (the batch without keys)


def test_nothing_is_written_outside_and_results_repeat(aj):
    """Outputs, workspace and the caller's buffers with canaries; a second run and a dirty workspace change no bit."""
    B, H, Hk, Lq, Lk, D = 2, 4, 2, 130, 3000, 128
    x = inputs(B, H, Hk, Lq, Lk, D)
    kl = torch.tensor([3000, 77], dtype=torch.int32, device="cuda")
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, k_lengths=kl)
    want = aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, k_lengths=kl)
    need = aj.attn_jvp_attention_bwd_workspace_bytes(B, H, Hk, Lq, Lk, D)
    pad = 512
    ws = torch.full((need + pad,), 255, dtype=torch.uint8, device="cuda")
    bufs = [torch.full((t.numel() + 2 * pad,), 7.0, dtype=torch.bfloat16, device="cuda") for t in want]
    a = aj.AttentionArgs()
    for n in ("q", "k", "v"):
        setattr(a, n, x[n].data_ptr())
        getattr(a, n + "_stride")[:] = x[n].stride()[:3]
    a.k_lengths = kl.data_ptr()
    a.B, a.H, a.Hk, a.Lq, a.Lk, a.D, a.causal, a.scale = B, H, Hk, Lq, Lk, D, 0, D ** -0.5
    outs = [b[pad:-pad] for b in bufs]
    stream = torch.cuda.current_stream().cuda_stream
    for _ in range(2):
        assert aj.attn_jvp_attention_bwd(a, x["d_o"], o, lse, *outs, ws, need, stream) == 0
        no_timeout(aj)
        for w, g, b in zip(want, outs, bufs):
            assert torch.equal(w.flatten(), g) and (b[:pad] == 7).all() and (b[-pad:] == 7).all()
        assert (ws[need:] == 255).all()


def test_unmasked_backward_is_the_sparse_one_of_all_blocks(aj):
    """Two roads to the same gradients, to rounding."""
    x = inputs(1, 3, 3, 700, 900, 128)
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True)
    sel = aj.block_selection(torch.ones(1, 3, 6, 8, dtype=torch.bool, device="cuda"), 700, 900)
    for a, b in zip(aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse),
                    aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel)):
        assert (a.double() - b.double()).norm() <= 5e-3 * b.double().norm()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(aj, D, causal):
    """Along d = g / |g| + r / 2 (r a random unit vector) the loss's central difference in 64 bits is <g, d>; the whole gradient is within
    1e-2 |g| (what a tensor's relative error may be), hence its product with d within 1.5e-2 |g|: a gradient that is zero, halved or short of a block fails."""
    B, H, Hk, L, lengths = 2, 4, 2, 260, [260, 150]
    x = inputs(B, H, Hk, L, L, D)
    kl = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, causal=causal, k_lengths=kl)
    got = dict(zip("qkv", aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, causal=causal, k_lengths=kl)))
    key, query = torch.arange(L, device="cuda"), torch.arange(L, device="cuda")[:, None]
    keep = (key < kl.view(B, 1, 1, 1)) & ((key <= query) if causal else True)
    full = {n: x[n].double() for n in "qkv"}

    def loss(t):
        kk, vv = (t[n].repeat_interleave(H // Hk, 2) for n in "kv")
        S = torch.where(keep, torch.einsum("bihd,bjhd->bhij", t["q"], kk) * D ** -0.5, -float("inf"))
        return (torch.einsum("bhij,bjhd->bihd", torch.softmax(S, -1), vv) * x["d_o"].double()).sum()

    leaves = {n: t.clone().requires_grad_() for n, t in full.items()}
    grads = dict(zip("qkv", torch.autograd.grad(loss(leaves), list(leaves.values()))))
    gen = torch.Generator(device="cuda").manual_seed(2)
    for n in "qkv":
        g = grads[n]
        for _ in range(2):
            r = torch.randn(g.shape, generator=gen, device="cuda", dtype=torch.float64)
            d = g / g.norm() + 0.5 * r / r.norm()
            e = 1e-4
            up, down = (loss({**full, n: full[n] + s * e * d}) for s in (1, -1))
            want = (up - down) / (2 * e)
            assert ((got[n].double() * d).sum() - want).abs() <= 1.5e-2 * g.norm() + 1e-6 * want.abs(), n


def test_streams_capture_and_two_calls_at_once(aj):
    x = inputs(2, 4, 2, 500, 700, 128)
    y = inputs(2, 4, 2, 300, 900, 64, seed=3)
    kl = torch.tensor([700, 333], dtype=torch.int32, device="cuda")

    def step(z, lengths=None, causal=False):
        o, _, lse = aj.attention_jvp(z["q"], z["k"], z["v"], fwd_only=True, causal=causal, k_lengths=lengths)
        return (o, lse, *aj.attention_backward(z["d_o"], z["q"], z["k"], z["v"], o, lse, causal=causal, k_lengths=lengths))

    want = step(x, kl), step(y, causal=True)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = []
        for s, call in zip(streams, (lambda: step(x, kl), lambda: step(y, causal=True))):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(call())
        no_timeout(aj)
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, kl)
    kl.copy_(torch.tensor([0, 500]))                     # (lengths are read when the graph runs)
    graph.replay()
    no_timeout(aj)
    assert all(torch.equal(u, v) for u, v in zip(got, step(x, kl)))


def test_refusals(aj):
    x = inputs(2, 4, 2, 100, 100, 64)
    kl = torch.tensor([100, 50], dtype=torch.int32, device="cuda")
    q, k, v = x["q"], x["k"], x["v"]
    fwd = lambda q=q, k=k, v=v, **kw: aj.attention_jvp(q, k, v, **{**dict(fwd_only=True, causal=True), **kw})
    o, _, lse = fwd()
    bwd = lambda d_o=x["d_o"], q=q, k=k, v=v, o=o, lse=lse, **kw: aj.attention_backward(d_o, q, k, v, o, lse, **{**dict(causal=True), **kw})
    bad_qkv = [dict(k=k[:, :, :1].expand(-1, -1, 3, -1)), dict(k=k[:, :50]), dict(v=v[:, :50]), dict(v=v[:, :, :1]), dict(q=q.float()), dict(q=q.cpu()), dict(k=k.half()), dict(q=q[0]),
               dict(q=q.transpose(2, 3)), dict(k=k[:, :, :1].expand(-1, -1, 2, -1)), dict(k=k[:1]), dict(q=q[:, :0]), dict(k=k[:, :0], v=v[:, :0]), dict(k_lengths=kl[:1]), dict(k_lengths=kl.long()),
               dict(k_lengths=kl.cpu()), dict(scale=float("inf")), dict(q=torch.zeros(2, 100, 4, 96, device="cuda").bfloat16(), k=torch.zeros(2, 100, 2, 96, device="cuda").bfloat16(), v=torch.zeros(2, 100, 2, 96, device="cuda").bfloat16())]
    for b in bad_qkv:
        with pytest.raises((ValueError, aj.AttnJvpError)):
            fwd(**b)
        with pytest.raises((ValueError, aj.AttnJvpError)):
            bwd(**b)
    for b in (dict(splits=2), dict(fwd_only=False), dict(fwd_only=False, tq=x["tq"], tk=x["tk"]), dict(fwd_only=False, tq=x["tq"][:, :50])):
        with pytest.raises((ValueError, aj.AttnJvpError)):
            fwd(**b)
    for b in (dict(d_o=None), dict(d_o=x["d_o"].transpose(0, 1)), dict(o=o[:, :50]), dict(lse=lse.double()), dict(lse=lse[:1]), dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, aj.AttnJvpError)):
            bwd(**b)
