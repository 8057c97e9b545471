"""The step between two branches of a DiT block: gate + residual + norm + modulation, fused (``attn_jvp_adaln_*``).

    u  = post_weight . post_norm(h),   x' = x + gate . u,   y = weight . norm(x') (1 + scale) + shift

A block calls it once per branch: y of one call is the input of the next attention or MLP branch, whose output is the
next call's h.  Forward, forward with tangents (the JVP mode of the generator step) and backward (the student step).
Argument marshalling only; the arithmetic runs in the CUDA library, there is no CPU path.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import attn_jvp as _binding

NORMS = {None: 0, "layer": 1, "rms": 2}


class AdaLNArgs(ctypes.Structure):
    """attn_jvp_adaln_t of include/attn_jvp.h."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "h", "gate", "scale", "shift", "weight", "post_weight", "tx", "th",
                                                "tgate", "tscale", "tshift")]
                + [(n + "_stride", ctypes.c_longlong) for n in ("gate", "scale", "shift", "tgate", "tscale", "tshift")]
                + [(n, ctypes.c_int) for n in ("B", "L", "C", "x_dtype", "norm", "post_norm")]
                + [("eps", ctypes.c_float)])


class AdaLNGrads(NamedTuple):
    """Gradients of ``adaln_jvp``; None where the input was None (``x`` always has one)."""
    x: torch.Tensor
    h: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]
    shift: Optional[torch.Tensor]
    weight: Optional[torch.Tensor]
    post_weight: Optional[torch.Tensor]


def attn_jvp_adaln_fwd(args: AdaLNArgs, x_new, y, tx_new, ty, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_adaln_fwd(ctypes.byref(args), p(x_new), p(y), p(tx_new), p(ty), p(cuda_stream))


def attn_jvp_adaln_bwd_workspace_bytes(B, L, C) -> int:
    return int(_binding.load().attn_jvp_adaln_bwd_workspace_bytes(int(B), int(L), int(C)))


def attn_jvp_adaln_bwd(args: AdaLNArgs, dx_new, dy, dx, dh, dgate, dscale, dshift, dweight, dpost_weight, workspace,
                       workspace_bytes, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_adaln_bwd(ctypes.byref(args), p(dx_new), p(dy), p(dx), p(dh), p(dgate), p(dscale),
                                              p(dshift), p(dweight), p(dpost_weight), p(workspace), int(workspace_bytes),
                                              p(cuda_stream))


def _tokens(t, name, shape, dtype, device):
    """Address of a tensor of tokens (or of a norm weight), checked."""
    if t.device != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device} of shape {tuple(shape)}")
    return t.data_ptr()


def _row(t, name, B, C, device):
    """Address and row stride of a modulation row per batch."""
    if t is None:
        return None, 0
    if t.device != device or t.dtype is not torch.float32 or t.shape != (B, C) or t.stride(1) != 1 and C > 1:
        raise ValueError(f"{name} must be fp32 of shape {(B, C)} on {device} with contiguous rows")
    return t.data_ptr(), t.stride(0) if B > 1 else 0


def _marshal(x, h, gate, scale, shift, weight, post_weight, norm, post_norm, eps, tangents=None) -> AdaLNArgs:
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 3:
        raise ValueError("x must be a CUDA tensor [B][L][C]")
    if norm not in NORMS or post_norm not in NORMS:
        raise ValueError(f"norm and post_norm are one of {list(NORMS)}")
    dev, shape, xt = x.device, x.shape, x.dtype
    B, L, C = shape
    if xt is not torch.bfloat16 and xt is not torch.float32 or not x.is_contiguous():
        raise ValueError("x must be contiguous, bf16 or fp32")
    if h is None and (gate is not None or post_weight is not None or post_norm is not None):
        raise ValueError("gate, post_norm and post_weight act on h, which is None")
    if norm is None and (scale is not None or shift is not None or weight is not None):
        raise ValueError("scale, shift and weight act on the norm's result, and norm is None")
    g, ld_g = _row(gate, "gate", B, C, dev)
    s, ld_s = _row(scale, "scale", B, C, dev)
    b, ld_b = _row(shift, "shift", B, C, dev)
    tx = th = tg = ts = tb = None
    ld_tg = ld_ts = ld_tb = 0
    if tangents is not None:
        tx, th, tg, ts, tb = tangents
        if tx is None or (th is None) != (h is None):
            raise ValueError("with tangents tx is required, and th exactly where h is given")
        if h is None and tg is not None or norm is None and (ts is not None or tb is not None):
            raise ValueError("a tangent of something that does not act")
        tx = _tokens(tx, "tx", shape, xt, dev)
        th = None if th is None else _tokens(th, "th", shape, torch.bfloat16, dev)
        tg, ld_tg = _row(tg, "tgate", B, C, dev)
        ts, ld_ts = _row(ts, "tscale", B, C, dev)
        tb, ld_tb = _row(tb, "tshift", B, C, dev)
    return AdaLNArgs(x.data_ptr(), None if h is None else _tokens(h, "h", shape, torch.bfloat16, dev), g, s, b,
                     None if weight is None else _tokens(weight, "weight", (C,), torch.float32, dev),
                     None if post_weight is None else _tokens(post_weight, "post_weight", (C,), torch.float32, dev),
                     tx, th, tg, ts, tb, ld_g, ld_s, ld_b, ld_tg, ld_ts, ld_tb, B, L, C, int(xt is torch.float32), NORMS[norm],
                     NORMS[post_norm], eps)


def _bf16_like(x, h):
    return torch.empty_like(h) if h is not None else torch.empty_like(x, dtype=torch.bfloat16)


def adaln_jvp(x, h=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, norm="layer", post_norm=None,
              eps=1e-6, tx=None, th=None, tgate=None, tscale=None, tshift=None):
    """x' = x + gate . post_weight . post_norm(h) and y = weight . norm(x') (1 + scale) + shift, with tangents if given.

    x: [B][L][C] CUDA bf16 or fp32; h: bf16 [B][L][C] or None (x' is x itself then); gate, scale, shift: fp32 [B][C] with
    any row stride (a slice of a [B][6][C] modulation, a broadcast row) or None; weight, post_weight: fp32 [C] or None;
    norm, post_norm: "layer", "rms" or None (norm=None: y is None).  C: a multiple of 8 up to 8192.  ``tx`` (type of x),
    ``th`` (bf16) and optionally tgate, tscale, tshift select the JVP mode.
    Returns (x', y, tx', ty); x', tx' have the type of x, y, ty are bf16; the tangents are None without ``tx``.
    """
    jvp = any(t is not None for t in (tx, th, tgate, tscale, tshift))
    a = _marshal(x, h, gate, scale, shift, weight, post_weight, norm, post_norm, eps,
                 (tx, th, tgate, tscale, tshift) if jvp else None)
    if h is None and norm is None:
        raise ValueError("neither h nor norm: nothing to compute")
    xn = None if h is None else torch.empty_like(x)
    y = None if norm is None else _bf16_like(x, h)
    txn = torch.empty_like(x) if jvp and h is not None else None
    ty = _bf16_like(x, h) if jvp and norm is not None else None
    _binding._call_on(x.device, attn_jvp_adaln_fwd, a, xn, y, txn, ty)
    return (x if h is None else xn), y, (tx if h is None else txn), ty


def adaln_backward(dx_new, dy, x, h=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, norm="layer",
                   post_norm=None, eps=1e-6, workspace=None) -> AdaLNGrads:
    """Gradients of ``adaln_jvp`` for dx' (type of x, or None: 0) and dy (bf16, or None: 0).

    The forward's inputs are passed again; its statistics are recomputed in the same pass.  Gradients of x have the type
    of x, of h bf16, of the modulation fp32 [B][C] (one row per sample also where the input's rows were shared), of the
    weights fp32 [C].  ``workspace``: a CUDA uint8 tensor of at least attn_jvp_adaln_bwd_workspace_bytes(B, L, C).
    """
    a = _marshal(x, h, gate, scale, shift, weight, post_weight, norm, post_norm, eps)
    if dx_new is not None:
        _tokens(dx_new, "dx_new", x.shape, x.dtype, x.device)
    if dy is not None:
        if norm is None:
            raise ValueError("dy given, but norm is None")
        _tokens(dy, "dy", x.shape, torch.bfloat16, x.device)
    B, L, C = x.shape
    dx = torch.empty_like(x)
    dh = None if h is None else torch.empty_like(h)

    # the gradients of the modulation and of the weights, one allocation
    rows = [C * B if t is not None and t.dim() == 2 else C if t is not None else 0 for t in (gate, scale, shift, weight, post_weight)]
    flat = x.new_empty(sum(rows), dtype=torch.float32).split(rows) if any(rows) else (None,) * 5
    dgate, dscale, dshift = (f.view(B, C) if n else None for f, n in zip(flat, rows[:3]))
    dw, dwp = (f if n else None for f, n in zip(flat[3:], rows[3:]))
    need = attn_jvp_adaln_bwd_workspace_bytes(B, L, C)
    if workspace is None:
        workspace, size = x.new_empty(need, dtype=torch.uint8), need
    elif workspace.device != x.device:
        raise ValueError(f"workspace must be on {x.device}")
    else:
        size = workspace.numel() * workspace.element_size()
    _binding._call_on(x.device, attn_jvp_adaln_bwd, a, dx_new, dy, dx, dh, dgate, dscale, dshift, dw, dwp, workspace, size)
    return AdaLNGrads(dx, dh, dgate, dscale, dshift, dw, dwp)
