"""How large the 2-norm of the errors of attention's gradients is to be expected from the roundings that the kernels make, row by row (test harness only).

A value that is rounded to bf16 is off by a variable of standard deviation ulp / sqrt 12; roundings of different values are taken as independent, so that their
squares add up:
  - dS and the result, and for dV P, are rounded to bf16 once each;
  - delta_i = dO_i . O_i takes O as the forward returned it.  O was rounded to bf16 (each channel), and the forward's products took the exponentials in bf16 (off by
    at most a half of 2^-7 of themselves: key j moves delta by that share of P_ij dP_ij).  An error e_i of delta moves dS_ij by P_ij e_i: dQ_i by
    s e_i sum_j P_ij k_j, dK_j by s P_ij e_i q_i.
fp32 sums are a 2^-24 and left out.  What delta adds grows with the size of O, not with the number of keys: rows whose probability lies at few keys have a large O
however many they see.
"""
import math

import torch

ROOM = 1.3        # the 2-norm of thousands of independent roundings against its expected value


def variance(x):
    """Of the rounding of x to bf16."""
    _, e = torch.frexp(x)
    return torch.where(x == 0, 0.0, torch.ldexp(torch.ones_like(x), 2 * (e - 8)) / 12)


def gradients(q, k, v, d_o, scale, causal=False, lengths=None, rounded_o=True):
    """{name: (gradient in 64 bits, expected 2-norm of its error)} of dq, dk, dv; rounded_o False: with an exact delta."""
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    out, square = dict(dq=z(q), dk=z(k), dv=z(v)), dict(dq=0.0, dk=0.0, dv=0.0)
    i = torch.arange(Lq, device=q.device)
    for b in range(B):
        n = Lk if lengths is None else max(0, min(Lk, int(lengths[b])))
        if n == 0:
            continue
        for h in range(H):
            hk = h // (H // Hk)
            Q, K, V, G = q[b, :, h].double(), k[b, :n, hk].double(), v[b, :n, hk].double(), d_o[b, :, h].double()
            S = Q @ K.T * scale
            if causal:
                S = torch.where(torch.arange(n, device=q.device) <= i[:, None] + (Lk - Lq), S, -math.inf)
            P = torch.where((S > -math.inf).any(-1, keepdim=True), torch.softmax(S, -1), 0.0)
            O, dP = P @ V, G @ V.T
            dS = P * (dP - (G * O).sum(-1, keepdim=True))
            out["dq"][b, :, h] = dS @ K * scale
            out["dk"][b, :n, hk] += dS.T @ Q * scale
            out["dv"][b, :n, hk] += P.T @ G
            q2, k2, rounds = Q.square().sum(-1), K.square().sum(-1), variance(dS)
            e2 = ((G.square() * variance(O)).sum(-1) + (P * dP).square().sum(-1) * 2.0 ** -14 / 12) * float(rounded_o)
            square["dq"] += scale ** 2 * ((rounds @ k2).sum() + (e2 * (P @ K).square().sum(-1)).sum())
            square["dk"] += scale ** 2 * ((rounds.T @ q2).sum() + (e2 * q2 * P.square().sum(-1)).sum())
            square["dv"] += (variance(P).T @ G.square().sum(-1)).sum()
    return {name: (g, math.sqrt(float(square[name] + variance(g).sum()))) for name, g in out.items()}


def check(got, want, what=""):
    """The gradients' errors in the 2-norm, each at most ROOM times what is expected; {name: error relative to the gradient}."""
    rel = {}
    for name, g in zip(("dq", "dk", "dv"), got):
        value, expected = want[name]
        off = (g.double() - value).norm().item()
        rel[name] = off / value.norm().item()
        assert off <= ROOM * expected, f"{what}{name}: {rel[name]:.2g} of the gradient, {off / expected:.3g} times the expected error"
    return rel
