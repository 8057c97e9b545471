"""Masked attention at the ends of its ranges: one query and many keys, many batches, one key head for many, outputs that are aligned to 16 bytes
only, one tensor in several places, strides along axes of one."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention import aj, inputs, no_timeout, run_all  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_one_query_and_many_keys(aj, D, causal):
    run_all(aj, inputs(2, 2, 1, 1, 60001, D), causal, [60001, 40000])
    run_all(aj, inputs(1, 1, 1, 40001, 1, D), causal)


@pytest.mark.parametrize("D", [64, 128])
def test_many_batches_and_many_heads(aj, D):
    run_all(aj, inputs(600, 1, 1, 3, 5, D), True, [b % 7 for b in range(600)])
    run_all(aj, inputs(1, 96, 1, 140, 150, D), True, [149])


@pytest.mark.parametrize("D", [64, 128])
def test_outputs_aligned_to_16_bytes(aj, D):
    B, H, Hk, Lq, Lk = 2, 2, 1, 150, 200
    x = inputs(B, H, Hk, Lq, Lk, D)
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, causal=True)
    want = aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, causal=True)
    a = aj.AttentionArgs()
    for n in "qkv":
        setattr(a, n, x[n].data_ptr())
        getattr(a, n + "_stride")[:] = x[n].stride()[:3]
    a.B, a.H, a.Hk, a.Lq, a.Lk, a.D, a.causal, a.scale = B, H, Hk, Lq, Lk, D, 1, D ** -0.5
    outs = [torch.full((t.numel() + 16,), 7.0, dtype=torch.bfloat16, device="cuda") for t in want]
    need = aj.attn_jvp_attention_bwd_workspace_bytes(B, H, Hk, Lq, Lk, D)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    at = [t[8:-8] for t in outs]
    assert aj.attn_jvp_attention_bwd(a, x["d_o"], o, lse, *at, ws, need, torch.cuda.current_stream().cuda_stream) == 0
    no_timeout(aj)
    for w, g, t in zip(want, at, outs):
        assert torch.equal(w.flatten(), g) and (t[:8] == 7).all() and (t[-8:] == 7).all()


@pytest.mark.parametrize("D", [64, 128])
def test_one_tensor_in_several_places(aj, D):
    """q = k = v = dO.  Held to the tolerance of every element, not to a share of the tensor's norm as independent tensors are: a query sees its own key
    with P near 1 (score |q|^2 / 8 = 8 at D = 64, the 100 others of size 1: 1 - P = 100 e^(1/2 - 8) = 0.055, for |q|^2 = 80 0.007), so dS = P (dP - delta) = P (1 - P) |q|^2
    is 3.3 to 0.6 while delta = dO . O, of size 64, carries the rounding of O to bf16: 0.6 2^-9 sqrt(sum (dO O)^2) = 0.6 2^-9 sqrt(64 . 3 . 0.8) = 0.0146 in the mean: 0.4 to 3 % of
    dS, and so of dQ.  The tolerances have that term."""
    x = inputs(2, 3, 3, 200, 200, D)
    q, tq, lengths = x["q"], x["tq"], [200, 90]
    ref = R.attention(q, q, q, D ** -0.5, True, lengths, tq, tq, tq, q)
    kw = dict(causal=True, k_lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    o, to, lse = aj.attention_jvp(q, q, q, tq, tq, tq, **kw)
    grads = aj.attention_backward(q, q, q, q, o, lse, **kw)
    no_timeout(aj)
    for n, got in zip(("o", "to", "lse", "dq", "dk", "dv"), (o, to, lse, *grads)):
        value, tol = ref[n]
        assert ((got.double() - value).abs() <= tol).all(), n


@pytest.mark.parametrize("D", [64, 128])
def test_strides_along_axes_of_one(aj, D):
    x = inputs(1, 1, 1, 1, 1, D)
    want = run_all(aj, x, True)
    y = dict(x, **{n: x[n].as_strided((1, 1, 1, D), (3, 5, 7, 1)) for n in "qkv"})
    for a, b in zip(run_all(aj, y, True, tangents=False), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
def test_peaked_rows(aj, D):
    """Scores of some hundreds to thousands: each row's probability is all at its own key (its score is ahead by more than 40), so o is that key's value, dv the
    row's gradient, lse the score.  p and the result are rounded once each (2^-8); a score of D products of one sign may be off by D 2^-23 of itself, which two passes
    may do differently and p takes in as e^that."""
    x = inputs(1, 2, 2, 256, 256, D)
    q = x["k"] * 8
    o, _, lse = aj.attention_jvp(q, x["k"], x["v"], fwd_only=True, causal=True, scale=1.0)
    dq, dk, dv = aj.attention_backward(x["d_o"], q, x["k"], x["v"], o, lse, causal=True, scale=1.0)
    no_timeout(aj)
    S = torch.einsum("bihd,bjhd->bhij", q.double(), x["k"].double())
    top = S.diagonal(dim1=2, dim2=3)
    others = S.masked_fill(torch.eye(256, dtype=torch.bool, device="cuda") | ~torch.ones_like(S, dtype=torch.bool).tril(), -float("inf")).amax(-1)
    assert (top - others > 40).all()
    assert ((lse.double() - top).abs() <= D * 2.0 ** -23 * top).all()
    off = (D * 2.0 ** -23 * top * 2).expm1().transpose(1, 2)[..., None] + 2.0 ** -7 + 2.0 ** -16
    for got, want in ((o, x["v"]), (dv, x["d_o"])):
        assert ((got.double() - want.double()).abs() <= off * want.double().abs() + 1e-6).all()
    assert torch.isfinite(dq).all() and torch.isfinite(dk).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,Lk,causal,lengths", [(600, 2, False, None), (600, 5, False, None), (600, 12, False, None), (600, 300, False, [3, 12]), (64, 64, True, None), (16, 16, True, None),
                                                  (700, 20, True, None), (40, 60, True, [60, 30])])
def test_rows_that_see_few_keys(aj, D, Lq, Lk, causal, lengths):
    """dS and the results are rounded to bf16 once each: relative roundings of 2^-9 / sqrt 3 = 0.0011 times the spread of a mantissa (1 to 2: the steps are 2^-8 of its lower end), 0.0017
    in the 2-norm, so 0.0024 for both and 0.0029 with a fifth of room; an o that was rounded before it went into delta would add up to 0.0027 in quadrature, 0.0036."""
    x = inputs(2, 4, 2, Lq, Lk, D)
    s = D ** -0.5
    kw = dict(causal=causal, k_lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    o, _, lse = aj.attention_jvp(x["q"], x["k"], x["v"], fwd_only=True, **kw)
    ref = R.attention(x["q"], x["k"], x["v"], s, causal, lengths, d_o=x["d_o"])
    grads = aj.attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, **kw)
    no_timeout(aj)
    for n, got in zip(("dq", "dk", "dv"), grads):
        rel = ((got.double() - ref[n][0]).norm() / ref[n][0].norm()).item()
        assert rel <= 0.0029, f"{n}: {rel:.2g}"
        R.check(n, got, ref[n])
