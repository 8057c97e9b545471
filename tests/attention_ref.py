"""64-bit statement of dense attention with a causal mask, key lengths and shared key heads, its tangent and its gradients, with
how far a kernel may be off; derivation and constants are those of tests/sparse_ref.py (test harness only).

Sums over the heads that share a key head are sums of their terms, and so are the tolerances of what goes into them; the
result is rounded once.
"""
import math

import torch

from tests.sparse_ref import A, SMALL, U, check  # noqa: F401


def attention(q, k, v, scale, causal=False, lengths=None, tq=None, tk=None, tv=None, d_o=None):
    """{name: (value, tolerance)}: o, lse, mu, to with tangents, dq, dk, dv with d_o.  lengths: a list, or None."""
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    names = ["o"] + (["to"] if tq is not None else []) + (["dq"] if d_o is not None else [])
    out = {n: (z(q), z(q) + 1e-30) for n in names}
    if d_o is not None:
        out.update(dk=(z(k), z(k) + 1e-30), dv=(z(k), z(k) + 1e-30))
    rows = torch.zeros(B, H, Lq, dtype=torch.float64, device=q.device)
    out["lse"], out["mu"] = (rows.clone() - math.inf, rows.clone()), (rows.clone(), rows.clone())
    i, s = torch.arange(Lq, device=q.device), abs(scale)
    for b in range(B):
        n = Lk if lengths is None else max(0, min(Lk, int(lengths[b])))
        if n == 0:
            continue
        keep = torch.ones(Lq, n, dtype=torch.bool, device=q.device)
        if causal:
            keep = torch.arange(n, device=q.device) <= i[:, None] + (Lk - Lq)
        some = keep.any(-1, keepdim=True)
        for h in range(H):
            hk = h // (H // Hk)
            Q, K, V = q[b, :, h].double(), k[b, :n, hk].double(), v[b, :n, hk].double()
            S = torch.where(keep, Q @ K.T * scale, -math.inf)
            lse = torch.logsumexp(S, -1)
            P = torch.where(some, torch.softmax(S, -1), 0.0)
            O = P @ V

            def put(name, value, tol):
                out[name][0][b, :, h], out[name][1][b, :, h] = value, tol

            put("o", O, (U + A) * (P @ V.abs()) + U * O.abs() + 1e-30)
            out["lse"][0][b, h], out["lse"][1][b, h] = lse, A / 10 * (1 + torch.where(some[:, 0], lse.abs(), 0.0))
            if tq is not None:
                T = tq[b, :, h].double()
                tS, tV, m = T @ K.T * scale, torch.zeros_like(V), (T.abs() @ K.abs().T) * s
                if tk is not None:
                    tK, tV = tk[b, :n, hk].double(), tv[b, :n, hk].double()
                    tS, m = tS + Q @ tK.T * scale, m + (Q.abs() @ tK.abs().T) * s
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
                dQ = dS @ K * scale
                put("dq", dQ, s * (e @ K.abs()) + U * dQ.abs() + 1e-30)
                for name, value, tol in (("dk", dS.T @ Q * scale, s * (e.T @ Q.abs())), ("dv", P.T @ G, (U + A) * (P.T @ G.abs()))):
                    out[name][0][b, :n, hk] += value
                    out[name][1][b, :n, hk] += tol
    if d_o is not None:
        for name in ("dk", "dv"):
            out[name][1].add_(U * out[name][0].abs())
    return out
