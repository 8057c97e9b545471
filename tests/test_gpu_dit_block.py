"""The new layers together, as a DiT block uses them: norm + modulation -> q, k, v -> QK norm -> sparse core -> projection ->
gate + residual + norm + modulation, in JVP mode and in training, against the same block in 64 bits.

Every bf16 tensor between two layers is rounded (half a step, 2^-9 in the mean of many elements, 2^-8 at most); the longest
path from an input to an output has y, q, normed q, P or dS, o, projected h and y again (seven), and a backward pass as many
once more.  Roundings of different elements are independent, so in the 2-norm they add up like sqrt(14) 2^-8 / sqrt(3) = 0.9 %
of magnitudes that the sums behind them may cancel down to a half; 3 % leaves that and no more.
"""
import pytest
import torch

from tests import adaln_ref

pytestmark = pytest.mark.gpu
REL = 0.03


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


B, L, H, D, TOPK = 2, 700, 4, 64, 3
C = H * D


def params(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s, sigma=1.0: torch.randn(*s, generator=g, device="cuda") * sigma  # noqa: E731
    return dict(x=rn(B, L, C), mod=rn(B, 6, C, sigma=0.3), wqkv=rn(C, 3 * C, sigma=C ** -0.5).bfloat16(),
                wo=rn(C, C, sigma=C ** -0.5).bfloat16(), tx=rn(B, L, C, sigma=0.5), tmod=rn(B, 6, C, sigma=0.1),
                dx=rn(B, L, C), dy=rn(B, L, C).bfloat16())


def reference(x, mod, wqkv, wo, mask):
    """64-bit block for a given selection; the attention core's q and k pass the RMS norm without weight."""
    s1, b1, g1, s2, b2, _ = mod.unbind(1)
    _, y = adaln_ref.step(x, None, None, s1, b1, None, None, "layer", None, 1e-6)
    q, k, v = ((y @ wqkv).view(B, L, 3, H, D)[:, :, i].transpose(1, 2) for i in range(3))
    q, k = (t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) for t in (q, k))
    keep = mask.repeat_interleave(128, 2)[:, :, :L].repeat_interleave(128, 3)[..., :L]
    p = torch.softmax((q @ k.transpose(-1, -2) * D ** -0.5).masked_fill(~keep, -float("inf")), -1)
    h = (p @ v).transpose(1, 2).reshape(B, L, C) @ wo
    return adaln_ref.step(x, h, g1, s2, b2, None, None, "layer", None, 1e-6)


def rel(got, ref):
    return ((got.double() - ref).norm() / ref.norm()).item()


def test_jvp_mode(aj):
    p = params()
    norm, core = aj.AdaLNJVP(C), aj.SparseAttentionCoreJVP(TOPK)
    s1, b1, g1, s2, b2, _ = zip(p["mod"].unbind(1), p["tmod"].unbind(1))
    (x, tx), (y, ty) = norm((p["x"], p["tx"]), scale=s1, shift=b1, withT=True)
    assert x is p["x"] and tx.data_ptr() == p["tx"].data_ptr()
    one = torch.ones(D, device="cuda")
    (q, k, v), (tq, tk, tv) = ([t.contiguous() for t in (u @ p["wqkv"]).view(B, L, 3, H, D).unbind(2)] for u in (y, ty))
    q, tq = aj.qknorm_jvp(q, tq, one)
    k, tk = aj.qknorm_jvp(k, tk, one)
    o, to = core((q, tq), (k, tk), (v, tv), withT=True)
    h, th = ((u.view(B, L, C) @ p["wo"]) for u in (o, to))
    (xn, txn), (yn, tyn) = norm((x, tx), (h, th), g1, s2, b2, withT=True)
    torch.cuda.synchronize()
    assert aj.attn_jvp_device_status() == 0
    mask = core.last_selection.mask
    f = lambda a, m: reference(a, m, p["wqkv"].double(), p["wo"].double(), mask)  # noqa: E731
    (rx, ry), (rtx, rty) = torch.func.jvp(f, (p["x"].double(), p["mod"].double()), (p["tx"].double(), p["tmod"].double()))
    for n, got, ref in (("x'", xn, rx), ("y", yn, ry), ("tx'", txn, rtx), ("ty", tyn, rty)):
        assert rel(got, ref) <= REL, (n, rel(got, ref))


def test_training(aj):
    p = params(1)
    norm, core = aj.AdaLNJVP(C), aj.SparseAttentionCoreJVP(TOPK)
    x, mod = p["x"].clone().requires_grad_(), p["mod"].clone().requires_grad_()
    wqkv, wo = p["wqkv"].clone().requires_grad_(), p["wo"].clone().requires_grad_()
    s1, b1, g1, s2, b2, _ = mod.unbind(1)
    x1, y = norm(x, scale=s1, shift=b1)
    q, k, v = (t.contiguous() for t in (y @ wqkv).view(B, L, 3, H, D).unbind(2))
    q, k = ((t.float() * torch.rsqrt(t.float().square().mean(-1, keepdim=True) + 1e-6)).bfloat16() for t in (q, k))
    o = core(q, k, v)
    xn, yn = norm(x1, o.view(B, L, C) @ wo, g1, s2, b2)
    torch.autograd.backward((xn, yn), (p["dx"], p["dy"]))
    torch.cuda.synchronize()
    assert aj.attn_jvp_device_status() == 0
    mask = core.last_selection.mask
    leaves = [t.detach().double().requires_grad_() for t in (x, mod, wqkv, wo)]
    rx, ry = reference(*leaves, mask)
    grads = torch.autograd.grad((rx, ry), leaves, (p["dx"].double(), p["dy"].double()))
    assert rel(xn.detach(), rx.detach()) <= REL and rel(yn.detach(), ry.detach()) <= REL
    for n, got, ref in zip(("x", "mod", "wqkv", "wo"), (x, mod, wqkv, wo), grads):
        assert rel(got.grad, ref) <= REL, (n, rel(got.grad, ref))


def test_learnt_norm_weights_and_parts_without_gradient(aj):
    """Parameters of the layer get their gradients; an unused output (y of the last block) costs none."""
    p = params(2)
    layer = aj.AdaLNJVP(C, norm="rms", post_norm="layer", affine=True, post_affine=True).cuda()
    with torch.no_grad():
        layer.weight += 0.1 * p["dx"][0, 0]
        layer.post_weight += 0.1 * p["dx"][0, 1]
    x, h = p["x"].clone().requires_grad_(), p["dy"].clone().requires_grad_()
    gate = p["mod"][:1, 0].expand(B, C).detach().requires_grad_()        # one row for every sample
    xn, y = layer(x, h, gate)
    (xn * p["dx"]).sum().backward()
    r = [t.detach().double().requires_grad_() for t in (x, h, gate, layer.post_weight)]
    rx, _ = adaln_ref.step(r[0], r[1], r[2], None, None, None, r[3], None, "layer", 1e-6)
    want = torch.autograd.grad((rx * p["dx"].double()).sum(), r)
    for got, ref in zip((x.grad, h.grad, gate.grad, layer.post_weight.grad), want):
        assert rel(got, ref) <= REL
    assert layer.weight.grad is None or not layer.weight.grad.any()
    assert y.shape == x.shape and y.dtype == torch.bfloat16


def test_selection_passed_in(aj):
    q, k, v = (torch.randn(1, 300, 2, 64, device="cuda").bfloat16().requires_grad_() for _ in range(3))
    core = aj.SparseAttentionCoreJVP(1)
    mask = torch.ones(1, 2, 3, 3, dtype=torch.bool, device="cuda")
    o = core(q, k, v, selection=aj.block_selection(mask, 300, 300))
    dense = aj.AttentionCoreJVP()(q.detach(), k.detach(), v.detach())
    assert rel(o.detach(), dense.double()) <= 0.01
    o.float().sum().backward()
    assert all(t.grad is not None and torch.isfinite(t.grad).all() for t in (q, k, v))
    with pytest.raises(ValueError):
        core((q, q), (k, k), v, withT=True)


@pytest.mark.parametrize("loss", [torch.sum, lambda t: t.square().sum()])
def test_no_second_derivatives(aj, loss):
    """A gradient of a gradient is an error, not a silent zero; the first gradients under create_graph are the usual ones."""
    x, h = (torch.randn(1, 20, 64, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    _, y = aj.AdaLNJVP(64)(x, h)
    (want,) = torch.autograd.grad(loss(y.float()), h, retain_graph=True)
    (g,) = torch.autograd.grad(loss(y.float()), h, create_graph=True)
    assert torch.equal(g, want)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (g.float().sum() + x.float().sum()).backward()
    q = torch.randn(1, 200, 2, 64, device="cuda").bfloat16().requires_grad_()
    (g,) = torch.autograd.grad(loss(aj.SparseAttentionCoreJVP(1)(q, q, q).float()), q, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (g.float().sum() + q.float().sum()).backward()


def test_a_mask_changed_before_the_backward_pass_is_an_error(aj):
    q = torch.randn(1, 300, 2, 64, device="cuda").bfloat16().requires_grad_()
    mask = torch.ones(1, 2, 3, 3, dtype=torch.bool, device="cuda")
    o = aj.SparseAttentionCoreJVP(1)(q, q, q, selection=aj.block_selection(mask, 300, 300))
    mask[0, 0, 0, 0] = False
    with pytest.raises(RuntimeError):
        o.float().sum().backward()


def test_frozen_inputs_get_no_gradient(aj):
    """Gradients go where they are asked for: a frozen stream, a frozen key."""
    p = params(4)
    layer = aj.AdaLNJVP(C).cuda()
    scale = p["mod"][:, 0].clone().requires_grad_()
    _, y = layer(p["x"], p["dy"], scale=scale)
    y.float().sum().backward()
    assert scale.grad.shape == (B, C) and p["x"].grad is None
    q, k, v = (torch.randn(1, 300, 2, 64, device="cuda").bfloat16() for _ in range(3))
    v.requires_grad_()
    aj.SparseAttentionCoreJVP(2)(q, k, v).float().sum().backward()
    assert v.grad is not None and q.grad is None and k.grad is None


def test_training_step_captured(aj):
    """Forward and backward of both layers in a CUDA graph, on a side stream, replayed on other inputs."""
    layer, core = aj.AdaLNJVP(C, norm="rms", affine=True).cuda(), aj.SparseAttentionCoreJVP(TOPK)

    def step(x, scale, dx):
        xn, y = layer(x, None, None, scale)
        q = y.view(B, L, H, D)
        o = core(q, q, q).reshape(B, L, C)
        _, z = layer(xn, o, None, scale)
        return (z.detach(), *torch.autograd.grad(z, (x, scale, layer.weight), dx))

    def args(seed):
        p = params(seed)
        return p["x"].requires_grad_(), p["mod"][:, 0].clone().requires_grad_(), p["dy"]

    a, b = args(1), args(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in step(*b)]
        step(*a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(*a)
    with torch.no_grad():
        for u, v in zip(a, b):
            u.copy_(v)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(got, want):
        assert torch.equal(u, v)
