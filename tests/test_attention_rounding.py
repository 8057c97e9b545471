"""The expected errors of tests/attention_rounding.py against a model of the kernels' roundings (CPU), and that what they allow is small: planted mistakes fail."""
import pytest
import torch

from tests import attention_rounding as E


def inputs(f, n, D, B=1, H=4, Hk=2, Lq=256, seed=0):
    g = torch.Generator().manual_seed(seed + n + D)
    rn = lambda *s, f=1.0: (torch.randn(*s, generator=g) * f).bfloat16()  # noqa: E731
    return rn(B, Lq, H, D, f=f), rn(B, n, Hk, D), rn(B, n, Hk, D), rn(B, Lq, H, D)


def modelled(q, k, v, d_o, s, exact_delta=False):
    """Gradients with bf16 where the kernels have it, sums in 64 bits.  The forward's reference lies up to 2^8 below the largest score."""
    r = lambda t: t.bfloat16().double()  # noqa: E731
    G = q.shape[2] // k.shape[2]
    Q, K, V, dO = (t.double().transpose(1, 2) for t in (q, k.repeat_interleave(G, 2), v.repeat_interleave(G, 2), d_o))
    S = Q @ K.transpose(-1, -2) * s
    low = S.amax(-1, keepdim=True) - torch.rand(S.shape[:-1] + (1,), generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 5
    X = torch.exp(S - low)
    P = X / X.sum(-1, keepdim=True)
    o = r(r(X) @ V / X.sum(-1, keepdim=True))
    dP = dO @ V.transpose(-1, -2)
    delta = (P * dP).sum(-1, keepdim=True) if exact_delta else (dO * o).sum(-1, keepdim=True)
    dS = r(P * (dP - delta))
    back = lambda t: t.unflatten(1, (-1, G)).sum(2).transpose(1, 2)  # noqa: E731
    dv, dk = back(r(P).transpose(-1, -2) @ dO), back(dS.transpose(-1, -2) @ Q) * s
    return r((dS @ K * s).transpose(1, 2)), r(dk), r(dv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [13, 64, 512])
@pytest.mark.parametrize("f", [1, 2, 4, 8])
def test_expected_errors(f, n, D):
    x = inputs(f, n, D)
    s = D ** -0.5
    for exact in (False, True):
        want = E.gradients(*x, s, rounded_o=not exact)
        got = modelled(*x, s, exact)
        E.check(got, want)
        for name, g in zip(("dq", "dk", "dv"), got):        # and no more than they need to allow
            assert (g - want[name][0]).norm() >= 0.6 * want[name][1], name


def test_mistakes_fail():
    """Among them what a test for finite values lets pass: zeros, halves, a missing delta, a block of keys or a head that is left out."""
    x = inputs(8, 512, 64)
    want = E.gradients(*x, 0.125)
    good = [t.double() for t in modelled(*x, 0.125)]
    E.check(good, want)
    dP_alone = [g.clone() for g in good]
    Q, K, V, G = (t.double().transpose(1, 2) for t in (x[0], x[1].repeat_interleave(2, 2), x[2].repeat_interleave(2, 2), x[3]))
    P = torch.softmax(Q @ K.transpose(-1, -2) * 0.125, -1)
    dP_alone[0] = ((P * (G @ V.transpose(-1, -2))) @ K * 0.125).transpose(1, 2)
    short = [g.clone() for g in good]
    short[1][:, 384:] = 0
    head = [g.clone() for g in good]
    head[0][:, :, 3] *= 1.02
    for bad in ([torch.zeros_like(g) for g in good], [good[0] / 2, *good[1:]], [good[0], good[1] / 2, good[2]], [good[0], good[1], -good[2]], dP_alone, short, head):
        with pytest.raises(AssertionError):
            E.check(bad, want)
