"""Gradients of attention whose probability lies at few of many keys: errors in the 2-norm against what the kernels' roundings let expect, and rows that are all at
one key."""
import pytest
import torch

from tests import attention_rounding as E
from tests.test_gpu_attention import aj, inputs, no_timeout  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(aj, x, factor, causal=False, lengths=None, rounded_o=True):
    q = (x["q"].float() * factor).bfloat16()
    s = q.shape[-1] ** -0.5
    kw = dict(causal=causal, k_lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    o, _, lse = aj.attention_jvp(q, x["k"], x["v"], fwd_only=True, **kw)
    got = aj.attention_backward(x["d_o"], q, x["k"], x["v"], o, lse, **kw)
    no_timeout(aj)
    return got, E.gradients(q, x["k"], x["v"], x["d_o"], s, causal, lengths, rounded_o)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [13, 64, 512, 4096])
@pytest.mark.parametrize("factor", [1, 2, 4, 8])
def test_queries_of_any_size(aj, D, n, factor):
    """Scores of spread 1 to 8: the largest probability of a row is 0.03 to 0.9 in the mean."""
    got, want = gradients(aj, inputs(2, 4, 2, 256, n, D), factor)
    rel = E.check(got, want)
    print("D", D, "keys", n, "factor", factor, {name: round(r, 5) for name, r in rel.items()})


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2, 5, 12])
@pytest.mark.parametrize("factor", [1, 2, 4, 8])
def test_few_keys(aj, D, n, factor):
    """Rows of at most 12 keys, whose delta is formed anew: the rounding of o adds nothing, whatever the size of the queries."""
    E.check(*gradients(aj, inputs(2, 4, 2, 256, n, D), factor, rounded_o=False))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("factor", [2, 6])
def test_masks(aj, D, factor):
    E.check(*gradients(aj, inputs(2, 4, 2, 400, 400, D), factor, True, [400, 150]))
    E.check(*gradients(aj, inputs(3, 4, 4, 500, 300, D), factor, False, [300, 0, 40]))


@pytest.mark.parametrize("D", [64, 128])
def test_rows_at_one_key(aj, D):
    """Scores of hundreds: a row's probability is all at its own key, whose score is ahead by more than 40, so that dS, dq and dk are 0 but for roundings.  o may be
    off from the key's value by the rounding of the exponential and its own (2^-8 each) and by what two passes make of a score of one sign (D 2^-23 of it, at most
    twice): so much of sum |dO v| may delta be off from dP, beside their sums in fp32 (D 2^-24 each); dS multiplies the key and the query."""
    x = inputs(1, 2, 2, 256, 256, D)
    q = x["k"] * 8
    o, _, lse = aj.attention_jvp(q, x["k"], x["v"], fwd_only=True, causal=True, scale=1.0)
    dq, dk, _ = aj.attention_backward(x["d_o"], q, x["k"], x["v"], o, lse, causal=True, scale=1.0)
    no_timeout(aj)
    Q, K, V, G = (t.double() for t in (q, x["k"], x["v"], x["d_o"]))
    S = torch.einsum("bihd,bjhd->bhij", Q, K)
    top = S.diagonal(dim1=2, dim2=3)
    others = S.masked_fill(torch.eye(256, dtype=torch.bool, device="cuda") | ~torch.ones_like(S, dtype=torch.bool).tril(), -float("inf")).amax(-1)
    assert (top - others > 40).all()
    two_passes = (D * 2.0 ** -23 * top * 2).expm1().transpose(1, 2)
    off = (two_passes + 2.0 ** -7 + 2.0 ** -16 + D * 2.0 ** -23) * (G * V).abs().sum(-1) * (1 + two_passes) * (1 + 2.0 ** -7)
    for name, got, size in (("dq", dq, K), ("dk", dk, Q)):
        assert (got.double().abs() <= off[..., None] * size.abs() + 1e-6).all(), name
