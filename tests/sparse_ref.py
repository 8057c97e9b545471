"""64-bit statement of attention over selected key blocks, its tangent and its gradients, with how far a kernel may be off
that rounds P, H~ and dS to bf16 as MMA operands and everything else in fp32 (test harness only).

Per element, with u = 2^-8 (half a bf16 step) and a = 2e-5 for the fp32 arithmetic in between: a score is a sum of D <= 128
products of bf16 values, off by at most 128 * 2^-24 = 8e-6 of sum |q||k|, which enters P as a relative error; the scores of
these tests stay below sum |q||k| s ~ 30, hence A = 5e-4 relative on P.
    O   : (u + A) sum P |v| + u |O|
    tS  : two sums of D products, off by a m, m = s sum (|tq||k| + |q||tk|) (256 * 2^-24 = 1.5e-5 < a), whatever is left of
          tS itself after cancellation; mu = sum P tS: 4 A max|tS| + a sum P m
    tO  : terms P (tS - c) v and P tv, c any value between the row's tS:
          (u + A) sum P (2 max|tS| |v| + |tv|) + a (sum P m |v| + max m sum P |v|) + u |tO|
    dV  : (u + A) sum P |dO| + u |dV|
    dS  : dS comes from P (off by A), dP (a of sum |dO||v|) and delta (off by u sum |dO||O|, since O is what the forward
          stored), and is rounded (u): e = (u + A) |dS| + P (a sum |dO||v| + (u + A) sum |dO||O|)
    dQ  : s sum e |k| + u |dQ|;   dK : s sum e |q| + u |dK|
"""
import math

import torch

U, A, SMALL = 2.0 ** -8, 5e-4, 2e-5
BLOCK = 128


def blocks(L):
    return -(-L // BLOCK)


def top_mask(q, k, topk):
    """Selection by mean-pooled scores in 64 bits, ties to the lower block."""
    qm = torch.stack([b.double().mean(1) for b in q.split(BLOCK, 1)], 1)
    km = torch.stack([b.double().mean(1) for b in k.split(BLOCK, 1)], 1)
    score = torch.einsum("bihd,bjhd->bhij", qm, km)
    rank = torch.sort(torch.sort(score, dim=-1, descending=True, stable=True).indices, dim=-1).indices
    return rank < topk


def attention(q, k, v, mask, scale, tq=None, tk=None, tv=None, d_o=None):
    """{name: (value, tolerance)}: o, lse, mu, to with tangents, dq, dk, dv with d_o."""
    B, Lq, H, D = q.shape
    Lk = k.shape[1]
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    out = {n: (z(q), z(q)) for n in (["o"] + (["to"] if tq is not None else []) + (["dq"] if d_o is not None else []))}
    if d_o is not None:
        out.update(dk=(z(k), z(k)), dv=(z(k), z(k)))
    rows = torch.zeros(B, H, Lq, dtype=torch.float64, device=q.device)
    out["lse"] = (rows.clone() - math.inf, rows.clone())
    out["mu"] = (rows.clone(), rows.clone())
    keep_all = mask.repeat_interleave(BLOCK, 2)[:, :, :Lq].repeat_interleave(BLOCK, 3)[..., :Lk]
    for b in range(B):
        for h in range(H):
            Q, K, V = q[b, :, h].double(), k[b, :, h].double(), v[b, :, h].double()
            keep = keep_all[b, h]
            some = keep.any(-1, keepdim=True)
            S = torch.where(keep, Q @ K.T * scale, -math.inf)
            lse = torch.logsumexp(S, -1)
            P = torch.where(some, torch.softmax(S, -1), 0.0)
            O = P @ V

            def put(name, value, tol):
                out[name][0][b, :, h], out[name][1][b, :, h] = value, tol

            put("o", O, (U + A) * (P @ V.abs()) + U * O.abs() + 1e-30)
            out["lse"][0][b, h], out["lse"][1][b, h] = lse, A / 10 * (1 + torch.where(some[:, 0], lse.abs(), 0.0))
            if tq is not None:
                tS = tq[b, :, h].double() @ K.T * scale
                tV = torch.zeros_like(V)
                m = (tq[b, :, h].double().abs() @ K.abs().T) * abs(scale)
                if tk is not None:
                    tS = tS + Q @ tk[b, :, h].double().T * scale
                    tV = tv[b, :, h].double()
                    m = m + (Q.abs() @ tk[b, :, h].double().abs().T) * abs(scale)
                top = torch.where(keep, tS.abs(), 0.0).amax(-1, keepdim=True)
                mu = (P * tS).sum(-1, keepdim=True)
                tO = (P * (tS - mu)) @ V + P @ tV
                m = torch.where(keep, m, 0.0)
                put("to", tO, (U + A) * (2 * top * (P @ V.abs()) + P @ tV.abs())
                    + SMALL * ((P * m) @ V.abs() + m.amax(-1, keepdim=True) * (P @ V.abs())) + U * tO.abs() + 1e-30)
                out["mu"][0][b, h], out["mu"][1][b, h] = mu[:, 0], 4 * A * top[:, 0] + SMALL * (P * m).sum(-1) + 1e-30
            if d_o is not None:
                G = d_o[b, :, h].double()
                dP = G @ V.T
                dS = P * (dP - (G * O).sum(-1, keepdim=True))
                e = (U + A) * dS.abs() + P * (SMALL * (G.abs() @ V.abs().T) + (U + A) * (G.abs() * O.abs()).sum(-1, keepdim=True))
                s = abs(scale)
                dQ, dK, dV = dS @ K * scale, dS.T @ Q * scale, P.T @ G
                put("dq", dQ, s * (e @ K.abs()) + U * dQ.abs() + 1e-30)
                put("dk", dK, s * (e.T @ Q.abs()) + U * dK.abs() + 1e-30)
                put("dv", dV, (U + A) * (P.T @ G.abs()) + U * dV.abs() + 1e-30)
    return out


def check(name, got, ref):
    value, tol = ref
    g = got.double()
    assert g.shape == value.shape, name
    inf = value == -math.inf
    assert torch.equal(g == -math.inf, inf), f"{name}: rows without keys"
    g, value, tol = g[~inf], value[~inf], tol[~inf]
    assert torch.isfinite(g).all(), f"{name}: non-finite"
    if g.numel():
        over = (g - value).abs() - tol
        assert over.max() <= 0, f"{name}: off by {(g - value).abs().max():.3g}, {over.max():.3g} over its tolerance"
        norm = value.norm()
        if value.numel() >= 4096 and norm > 0 and name != "lse":
            # over many elements roundings do not line up: a few half steps of 2^-9 in the mean
            assert (g - value).norm() <= 1e-2 * norm, f"{name}: relative error {(g - value).norm() / norm:.3g}"
