"""Gradients as autograd hands them to the layers: slices of a larger tensor that start anywhere in memory, and expanded ones."""
import pytest
import torch

from tests.test_gpu_attention import aj, no_timeout  # noqa: F401

pytestmark = pytest.mark.gpu


def rn(*shape):
    return torch.randn(*shape, device="cuda").bfloat16()


def layers(aj):
    """(name, outputs as a function of leaves, leaves) of every layer with autograd."""
    B, L, H, D = 2, 70, 2, 64
    table = aj.rotary_table(torch.arange(L, device="cuda"), D)
    dense, sparse, rotary, norm = aj.AttentionCoreJVP(causal=True), aj.SparseAttentionCoreJVP(topk=1), aj.QKRotaryJVP(D).cuda(), aj.AdaLNJVP(512).cuda()
    heads = [rn(B, L, H, D) for _ in range(3)]
    return [("attention", lambda q, k, v: (dense(q, k, v),), heads), ("selected blocks", lambda q, k, v: (sparse(q, k, v),), heads),
            ("rotary", lambda q, k: rotary(q, k, table), heads[:2]),
            ("adaLN", lambda x, h: norm(x, h, None, torch.zeros(B, 512, device="cuda"), torch.zeros(B, 512, device="cuda")), [rn(B, L, 512), rn(B, L, 512)])]


@pytest.mark.parametrize("which", range(4))
def test_gradients_that_start_anywhere(aj, which):
    """Outputs joined behind one more number: their gradients are slices whose first element lies 2 bytes behind an aligned one."""
    name, call, leaves = layers(aj)[which]
    xs = [t.clone().requires_grad_() for t in leaves]
    outs = call(*xs)
    weights = [torch.randn_like(o) for o in outs]
    want = torch.autograd.grad(outs, xs, weights)
    outs = call(*xs)
    joined = torch.cat([t for o in outs for t in (o.new_zeros(1), o.flatten())])
    w = torch.cat([t for g in weights for t in (g.new_zeros(1), g.flatten())])
    seen = []
    for o in outs:
        o.register_hook(lambda g: seen.append(g.data_ptr() % 16))
    got = torch.autograd.grad(joined, xs, w)
    no_timeout(aj)
    assert any(seen), name
    for a, b in zip(got, want):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("which", range(4))
def test_expanded_gradients(aj, which):
    """What a sum hands back: one number for all elements."""
    name, call, leaves = layers(aj)[which]
    xs = [t.clone().requires_grad_() for t in leaves]
    got = torch.autograd.grad([o.sum() for o in call(*xs)], xs)
    outs = call(*xs)
    for a, b in zip(got, torch.autograd.grad(outs, xs, [torch.ones_like(o) for o in outs])):
        assert torch.equal(a, b), name
    no_timeout(aj)
