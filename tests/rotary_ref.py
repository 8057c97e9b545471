"""Rotary tables and the per-head norm and rotation in 64 bits (test harness only)."""
import math

import torch

EPS = 1e-6


def table(positions, dims, base=10000.0, scaling=None, factor=1.0, original_length=None):
    """fp64 [...][R / 2][2] of positions [...][axes]."""
    out, size = [], 1.0
    for a, d in enumerate(dims):
        b, s = (v[a] if isinstance(v, (tuple, list)) else v for v in (base, factor))
        if scaling == "ntk":
            b = b * s ** (d / (d - 2))
        theta = torch.tensor([b ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64, device=positions.device)
        if scaling == "linear":
            theta = theta / s
        if scaling == "yarn":
            g = ((original_length * theta / (2 * math.pi) - 1) / 31).clamp(0, 1)
            theta = (1 - g) * theta / s + g * theta
        out.append(positions[..., a, None].double() * theta)
    if scaling == "yarn":
        s = factor[0] if isinstance(factor, (tuple, list)) else factor
        size = 0.1 * math.log(s) + 1
    angle = torch.cat(out, -1)
    return torch.stack([angle.cos(), angle.sin()], -1) * size


def rows_of(table, index, B, L):
    """The table row of every token: [B][L][R / 2][2]."""
    t = (table if table.dim() == 4 else table.expand(B, -1, -1, -1)).double()
    i = torch.arange(L, device=t.device).expand(B, L) if index is None else index.long().expand(B, L).clamp(0, t.shape[1] - 1)
    return torch.stack([t[b, i[b]] for b in range(B)])


def turn(u, cs, layout):
    R = 2 * cs.shape[-2]
    c, s = cs[..., 0].unsqueeze(-2), cs[..., 1].unsqueeze(-2)
    a, b = (u[..., :R // 2], u[..., R // 2:R]) if layout == "half" else (u[..., 0:R:2], u[..., 1:R:2])
    x, y = a * c - b * s, b * c + a * s
    turned = torch.cat([x, y], -1) if layout == "half" else torch.stack([x, y], -1).flatten(-2)
    return torch.cat([turned, u[..., R:]], -1)


def head(x, cs, w, b, norm, layout, eps=EPS):
    """y of x [B][L][H][D] for table rows cs [B][L][R / 2][2]; everything fp64."""
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    if norm is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        x = x * w
    if b is not None:
        x = x + b
    return turn(x, cs, layout)
