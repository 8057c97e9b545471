"""Gradients of the norms' weights and biases against the sizes of their own terms: dw_c = sum du_c n_c, db_c = sum du_c over batches, tokens and heads."""
import pytest
import torch

from tests import rotary_ref as R
from tests.test_gpu_rotary import aj, inputs  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [(1, 1, 1, 1, 128, 128, "interleaved", "rms"), (2, 333, 5, 1, 128, 128, "interleaved", "rms"), (3, 257, 6, 3, 64, 32, "half", "layer"),
         (1, 1025, 3, 3, 64, 64, "interleaved", "layer"), (1, 517, 12, 12, 128, 8, "interleaved", None), (2, 700, 16, 4, 128, 104, "half", "layer"),
         (1, 4000, 40, 40, 128, 128, "half", "rms")]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_sums(aj, case):
    """A term is off by at most the roundings behind it: three of du = dy cos + dy' sin, some twenty of n (a mean and a mean square over lanes, the root, the
    products), one of the product.  A sum adds at most 160 of them one after the other: the rows of a group of lanes (up to 80 here), 32 groups of a block, and
    in the join 10 blocks in a row and 32 rows.  340 steps of 2^-24 of the terms' sizes hold both with room."""
    B, L, H, Hk, D, Rt, layout, norm = case
    x = inputs(B, L, H, Hk, D, Rt, False, 0, False, True, True)
    kw = dict(norm=norm, layout=layout, **{n: x[n] for n in ("q_weight", "k_weight", "q_bias", "k_bias")})
    grads = aj.qk_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["table"], **kw)
    cs = R.rows_of(x["table"], x["index"], B, L)
    back = cs * torch.tensor([1.0, -1.0], device="cuda", dtype=torch.float64)
    for n in "qk":
        v, dy = x[n].double(), x["d" + n].double()
        mean = v.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(v[..., :1])
        r = torch.ones_like(mean) if norm is None else 1 / torch.sqrt((v - mean).square().mean(-1, keepdim=True) + R.EPS)
        normed, du = (v - mean) * r, R.turn(dy, back, layout)
        # |a| |cos| + |b| |sin| for either of a pair: the turn of the sizes with the sign of its difference taken away
        size = torch.maximum(R.turn(dy.abs(), back.abs(), layout).abs(), R.turn(dy.abs(), back.abs() * torch.tensor([1.0, -1.0], device="cuda", dtype=torch.float64), layout).abs())
        for m, got, want, terms in (("weight", getattr(grads, n + "_weight"), du * normed, size * (v.abs() + mean.abs()) * r),
                                    ("bias", getattr(grads, n + "_bias"), du, size)):
            want, terms = want.sum((0, 1, 2)), terms.sum((0, 1, 2))
            off = (got.double() - want).abs()
            assert (off <= 2.0 ** -24 * 340 * terms).all(), (n, m, (off / terms).max().item() * 2 ** 24)
