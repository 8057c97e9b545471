"""64-bit statement of the fused gate + residual + norm + modulation step, for the tests (test harness only)."""
import torch


def normed(v, kind, eps):
    if kind is None:
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)


def step(x, h, gate, scale, shift, w, wp, norm, post, eps):
    """x' and y for fp64 tensors; None where something is left out."""
    xn = x
    if h is not None:
        u = normed(h, post, eps)
        if wp is not None:
            u = u * wp
        if gate is not None:
            u = u * gate[:, None]
        xn = x + u
    if norm is None:
        return xn, None
    y = normed(xn, norm, eps)
    if w is not None:
        y = y * w
    if scale is not None:
        y = y * (1 + scale[:, None])
    if shift is not None:
        y = y + shift[:, None]
    return xn, y
