"""The comparison of gradients with differences: it accepts the 64-bit gradients and refuses ones with a mistake in them (CPU)."""
import pytest
import torch

from tests import sparse_differences as F
from tests import sparse_ref as R

SCALE = 64 ** -0.5


@pytest.fixture(scope="module")
def case():
    g = torch.Generator().manual_seed(3)
    x = {n: torch.randn(2, L, 2, 64, generator=g).bfloat16() for n, L in (("q", 150), ("k", 300), ("v", 300), ("d_o", 150))}
    mask = torch.tensor([[1, 0, 1], [1, 1, 1]], dtype=torch.bool).expand(2, 2, 2, 3).clone()
    r = R.attention(x["q"], x["k"], x["v"], mask, SCALE, d_o=x["d_o"])
    return x, mask, {n: r["d" + n][0] for n in "qkv"}


def test_the_gradients_pass(case):
    x, mask, grads = case
    assert F.passes(F.compare(grads, x, mask, SCALE)) == {"q", "k", "v"}
    rounded = {n: g.bfloat16() for n, g in grads.items()}
    assert F.passes(F.compare(rounded, x, mask, SCALE)) == {"q", "k", "v"}


def without_a_block(g):
    g = g.clone()
    g[:, :128] = 0
    return g


@pytest.mark.parametrize("mistake", [torch.zeros_like, torch.neg, lambda g: g / 2, lambda g: 1.1 * g, without_a_block,
                                     lambda g: g.flip(2), lambda g: g.roll(1, 1)],
                         ids=["zero", "sign", "half", "scale", "block", "heads", "rows"])
def test_mistakes_do_not_pass(case, mistake):
    x, mask, grads = case
    assert F.passes(F.compare({n: mistake(g) for n, g in grads.items()}, x, mask, SCALE)) == set()


def test_missing_terms_do_not_pass(case):
    """dS without delta, and the gradients of attention over all blocks."""
    x, mask, grads = case
    Q, K, V, G = (x[n].double().transpose(1, 2) for n in ("q", "k", "v", "d_o"))
    keep = mask.repeat_interleave(128, 2)[:, :, :150].repeat_interleave(128, 3)[..., :300]
    P = torch.softmax(torch.where(keep, Q @ K.transpose(-1, -2) * SCALE, -float("inf")), -1)
    dS = P * (G @ V.transpose(-1, -2)) * SCALE
    wrong = dict(q=(dS @ K).transpose(1, 2), k=(dS.transpose(-1, -2) @ Q).transpose(1, 2), v=grads["v"])
    assert F.passes(F.compare(wrong, x, mask, SCALE)) == {"v"}
    r = R.attention(x["q"], x["k"], x["v"], torch.ones_like(mask), SCALE, d_o=x["d_o"])
    assert F.passes(F.compare({n: r["d" + n][0] for n in "qkv"}, x, mask, SCALE)) == set()
