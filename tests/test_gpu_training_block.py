"""The operators of an attention branch in training, as a user runs them together: slices of a fused projection, rotary table, norm and
rotation of the heads, dense attention with shared key heads and padded contexts, their gradients, and the same branch in JVP mode.

Tolerances: every operator rounds its bf16 results once (2^-9 relative in the mean, 2^-8 at most); a branch of projections, rotation, attention and
their backward chain has some ten such roundings one after the other, none amplified by more than a small factor: relative errors of whole tensors stay below 2e-2.
"""
import pytest
import torch

from tests import rotary_ref as RR

pytestmark = pytest.mark.gpu
B, L, H, HK, D, RT = 2, 300, 4, 2, 64, 48


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def parts(aj, causal, context):
    g = torch.Generator(device="cuda").manual_seed(11)
    rn = lambda *s, f=1.0: (torch.randn(*s, generator=g, device="cuda") * f).bfloat16()
    C = H * D
    p = dict(x=rn(B, L, C), tx=rn(B, L, C), dy=rn(B, L, C), w=rn(C, (H + 2 * HK) * D, f=C ** -0.5), wo=rn(C, C, f=C ** -0.5))
    p["pos"] = torch.stack([torch.arange(L, device="cuda") // 20, torch.arange(L, device="cuda") % 20], -1).int()
    p["table"] = aj.rotary_table(p["pos"], (16, 32), base=(100.0, 10000.0))
    p["lengths"] = torch.tensor([L, 170], dtype=torch.int32, device="cuda") if context else None
    rot = aj.QKRotaryJVP(D).cuda()
    with torch.no_grad():
        for w in rot.parameters():
            w.add_(0.2 * torch.randn(D, generator=g, device="cuda"))
    return p, rot, aj.AttentionCoreJVP(causal=causal)


def branch(p, rot, core, x, w, wo):
    y = (x @ w).view(B, L, H + 2 * HK, D)
    q, k = rot(y[:, :, :H], y[:, :, H:H + HK], p["table"])
    return core(q, k, y[:, :, H + HK:], k_lengths=p["lengths"]).flatten(2) @ wo


def statement(p, rot, causal, x, w, wo, qw, kw):
    y = (x @ w).view(B, L, H + 2 * HK, D)
    cs = RR.table(p["pos"], (16, 32), base=(100.0, 10000.0)).expand(B, -1, -1, -1)
    q, k = RR.head(y[:, :, :H], cs, qw, None, "rms", "interleaved"), RR.head(y[:, :, H:H + HK], cs, kw, None, "rms", "interleaved")
    k, v = (t.repeat_interleave(H // HK, 2) for t in (k, y[:, :, H + HK:]))
    i = torch.arange(L, device="cuda")
    keep = torch.ones(B, 1, L, L, dtype=torch.bool, device="cuda")
    if causal:
        keep = keep & (i <= i[:, None])
    if p["lengths"] is not None:
        keep = keep & (i < p["lengths"].view(B, 1, 1, 1))
    S = torch.einsum("bihd,bjhd->bhij", q, k).masked_fill(~keep, -float("inf")) * D ** -0.5
    return torch.einsum("bhij,bjhd->bihd", torch.softmax(S, -1), v).flatten(2) @ wo


def near(name, got, want):
    rel = ((got.double() - want).norm() / want.norm()).item()
    assert rel <= 2e-2, f"{name}: relative error {rel:.3g}"


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("context", [False, True])
def test_training(aj, causal, context):
    p, rot, core = parts(aj, causal, context)
    leaves = [p[n].clone().requires_grad_() for n in ("x", "w", "wo")]
    z = branch(p, rot, core, *leaves)
    grads = torch.autograd.grad(z, (*leaves, rot.q_weight, rot.k_weight), p["dy"])
    exact = [t.detach().double().requires_grad_() for t in (*leaves, rot.q_weight, rot.k_weight)]
    want = statement(p, rot, causal, *exact)
    near("output", z, want)
    for n, a, b in zip(("x", "w", "wo", "q_weight", "k_weight"), grads, torch.autograd.grad(want, exact, p["dy"].double())):
        near(n, a, b)
    torch.cuda.synchronize()
    assert aj.attn_jvp_device_status() == 0


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("context", [False, True])
def test_jvp_mode(aj, causal, context):
    p, rot, core = parts(aj, causal, context)
    y, ty = ((t @ p["w"]).view(B, L, H + 2 * HK, D) for t in (p["x"], p["tx"]))
    q, k = rot((y[:, :, :H], ty[:, :, :H]), (y[:, :, H:H + HK], ty[:, :, H:H + HK]), p["table"], withT=True)
    o, to = core(q, k, (y[:, :, H + HK:], ty[:, :, H + HK:].contiguous()), withT=True, k_lengths=p["lengths"])
    z, tz = o.flatten(2) @ p["wo"], to.flatten(2) @ p["wo"]
    f = lambda x: statement(p, rot, causal, x, *(t.detach().double() for t in (p["w"], p["wo"], rot.q_weight, rot.k_weight)))
    want, twant = torch.func.jvp(f, (p["x"].double(),), (p["tx"].double(),))
    near("output", z, want)
    near("tangent", tz, twant)
    assert not z.requires_grad and core.last_lse.shape == (B, H, L)


def test_training_step_in_a_graph(aj):
    p, rot, core = parts(aj, True, True)

    def step():
        leaves = [p[n].detach().requires_grad_() for n in ("x", "w", "wo")]
        z = branch(p, rot, core, *leaves)
        return (z.detach(), *torch.autograd.grad(z, (*leaves, rot.q_weight, rot.k_weight), p["dy"]))

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_dense_core_is_differentiable_once(aj):
    q, k, v = (torch.randn(1, 200, 2, 64, device="cuda").bfloat16().requires_grad_() for _ in range(3))
    core = aj.AttentionCoreJVP()
    o = core(q, k, v)
    plain, _, lse = aj.attention_jvp(q.detach(), k.detach(), v.detach(), fwd_only=True)
    assert torch.equal(o, plain) and torch.equal(core.last_lse, lse) and o.requires_grad and not core.last_lse.requires_grad
    d_o = torch.randn(200, 2, 64, device="cuda").bfloat16().expand(1, -1, -1, -1)
    for a, b in zip(torch.autograd.grad(o, (q, k, v), d_o, retain_graph=True), aj.attention_backward(d_o.contiguous(), q.detach(), k.detach(), v.detach(), plain, lse)):
        assert torch.equal(a, b)
    (only,) = torch.autograd.grad(core(q.detach(), k, v.detach()), k, d_o)
    assert torch.isfinite(only).all()
    (g,) = torch.autograd.grad(core(q, k, v).float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()
    lengths = torch.tensor([100], dtype=torch.int32, device="cuda")
    z = core(q, k, v, k_lengths=lengths)
    lengths.add_(1)
    with pytest.raises(RuntimeError):
        z.float().sum().backward()
