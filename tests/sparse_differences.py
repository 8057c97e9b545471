"""Gradients of attention over selected key blocks against central differences of the 64-bit loss (test harness only).

A gradient g is compared with the loss's difference along directions that it has a large part in: d = g / |g| + r / 2, r a random
unit vector, so that <g, d> is about |g|.  With |got - g| <= 1e-2 |g|, the bound that tests/sparse_ref.py puts on the relative error of
a whole tensor, |<got, d> - <g, d>| <= 1e-2 |g| |d|, and |d| <= 1.5: the tolerance is at most 3 % of the smallest <g, d> = |g| / 2
that a direction can have, so a gradient that is zero, of the wrong sign, halved or short of a key block does not pass.  (Along
purely random directions the same bound would be several times as large as what is measured.)  The difference itself is
off by e^2 / 6 of a third derivative and by 2^-52 / e of the loss: below 1e-6 of it at e = 1e-4.
"""
import torch

from tests import sparse_ref as R

E = 1e-4


def loss(q, k, v, d_o, mask, scale):
    """sum O . dO in 64 bits; [B][L][H][D], every query block keeps something."""
    keep = mask.repeat_interleave(R.BLOCK, 2)[:, :, :q.shape[1]].repeat_interleave(R.BLOCK, 3)[..., :k.shape[1]]
    S = torch.where(keep, torch.einsum("bihd,bjhd->bhij", q, k) * scale, -float("inf"))
    return (torch.einsum("bhij,bjhd->bihd", torch.softmax(S, -1), v) * d_o).sum()


def compare(grads, x, mask, scale, draws=3):
    """[(name, <gradient, d>, difference along d, tolerance)] for grads = {"q": dq, "k": dk, "v": dv}."""
    full = {n: x[n].double() for n in ("q", "k", "v", "d_o")}
    ref = R.attention(x["q"], x["k"], x["v"], mask, scale, d_o=x["d_o"])
    gen = torch.Generator().manual_seed(5)
    out = []
    for n, got in grads.items():
        g = ref["d" + n][0]
        for _ in range(draws):
            r = torch.randn(g.shape, generator=gen, dtype=torch.float64).to(g.device)
            d = g / g.norm() + 0.5 * r / r.norm()
            up, down = (loss(**{**full, n: full[n] + s * E * d}, mask=mask, scale=scale) for s in (1, -1))
            out.append((n, (got.double() * d).sum().item(), ((up - down) / (2 * E)).item(), (1e-2 * g.norm() * d.norm()).item()))
    return out


def passes(rows):
    """Names whose every direction is within its tolerance."""
    assert all(tol <= 0.03 * abs(want) for _, _, want, tol in rows)
    return {n for n, *_ in rows} - {n for n, got, want, tol in rows if abs(got - want) > tol + 1e-6 * abs(want)}
