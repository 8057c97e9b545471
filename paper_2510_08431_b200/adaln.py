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
    return int(_binding.load().attn_jvp_adaln_fwd(ctypes.byref(args), p(x_new), p(y), p(tx_new), p(ty), p(cuda_stream)))


def attn_jvp_adaln_bwd_workspace_bytes(B, L, C) -> int:
    return int(_binding.load().attn_jvp_adaln_bwd_workspace_bytes(int(B), int(L), int(C)))


def attn_jvp_adaln_bwd(args: AdaLNArgs, dx_new, dy, dx, dh, dgate, dscale, dshift, dweight, dpost_weight, workspace,
                       workspace_bytes, cuda_stream) -> int:
    p = _binding._ptr
    return int(_binding.load().attn_jvp_adaln_bwd(ctypes.byref(args), p(dx_new), p(dy), p(dx), p(dh), p(dgate), p(dscale),
                                                  p(dshift), p(dweight), p(dpost_weight), p(workspace),
                                                  int(workspace_bytes), p(cuda_stream)))


def _tokens(t, name, shape, dtypes, device):
    if not t.is_cuda or t.device != device or t.dtype not in dtypes or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on {device} of shape {shape} and type {' or '.join(map(str, dtypes))}")


def _marshal(x, h, gate, scale, shift, weight, post_weight, norm, post_norm, eps, tangents=None) -> AdaLNArgs:
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 3:
        raise ValueError("x must be a CUDA tensor [B][L][C]")
    if norm not in NORMS or post_norm not in NORMS:
        raise ValueError(f"norm and post_norm are one of {list(NORMS)}")
    dev, shape = x.device, tuple(x.shape)
    B, L, C = shape
    _tokens(x, "x", shape, (torch.bfloat16, torch.float32), dev)
    a = AdaLNArgs(B=B, L=L, C=C, x_dtype=int(x.dtype == torch.float32), norm=NORMS[norm], post_norm=NORMS[post_norm], eps=eps)
    a.x = x.data_ptr()
    if h is not None:
        _tokens(h, "h", shape, (torch.bfloat16,), dev)
        a.h = h.data_ptr()
    elif gate is not None or post_weight is not None or post_norm is not None:
        raise ValueError("gate, post_norm and post_weight act on h, which is None")
    if norm is None and (scale is not None or shift is not None or weight is not None):
        raise ValueError("scale, shift and weight act on the norm's result, and norm is None")
    tx, th, tgate, tscale, tshift = tangents if tangents is not None else (None,) * 5
    rows = dict(gate=gate, scale=scale, shift=shift, tgate=tgate, tscale=tscale, tshift=tshift)
    for name, t in rows.items():
        if t is None:
            continue
        if t.device != dev or t.dtype != torch.float32 or tuple(t.shape) != (B, C) or (C > 1 and t.stride(1) != 1):
            raise ValueError(f"{name} must be fp32 of shape {(B, C)} on {dev} with contiguous rows")
        setattr(a, name, t.data_ptr())
        setattr(a, name + "_stride", t.stride(0) if B > 1 else 0)
    for name, t in dict(weight=weight, post_weight=post_weight).items():
        if t is not None:
            _tokens(t, name, (C,), (torch.float32,), dev)
            setattr(a, name, t.data_ptr())
    if tangents is not None:
        if tx is None or (th is None) != (h is None):
            raise ValueError("with tangents tx is required, and th exactly where h is given")
        if h is None and tgate is not None or norm is None and (tscale is not None or tshift is not None):
            raise ValueError("a tangent of something that does not act")
        _tokens(tx, "tx", shape, (x.dtype,), dev)
        a.tx = tx.data_ptr()
        if th is not None:
            _tokens(th, "th", shape, (torch.bfloat16,), dev)
            a.th = th.data_ptr()
    return a


def _raise(rc):
    if rc != 0:
        raise _binding.AttnJvpError(rc, _binding.attn_jvp_strerror(rc))


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
    y_like = dict(dtype=torch.bfloat16, device=x.device)
    xn = None if h is None else torch.empty_like(x)
    y = None if norm is None else torch.empty(x.shape, **y_like)
    txn = torch.empty_like(x) if jvp and h is not None else None
    ty = torch.empty(x.shape, **y_like) if jvp and norm is not None else None
    with torch.cuda.device(x.device):
        _raise(attn_jvp_adaln_fwd(a, xn, y, txn, ty, torch.cuda.current_stream().cuda_stream))
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
        _tokens(dx_new, "dx_new", tuple(x.shape), (x.dtype,), x.device)
    if dy is not None:
        if norm is None:
            raise ValueError("dy given, but norm is None")
        _tokens(dy, "dy", tuple(x.shape), (torch.bfloat16,), x.device)
    B, L, C = x.shape
    dx = torch.empty_like(x)
    dh = None if h is None else torch.empty_like(h)

    def row(t, *shape):
        return None if t is None else torch.empty(shape, dtype=torch.float32, device=x.device)

    dgate, dscale, dshift = row(gate, B, C), row(scale, B, C), row(shift, B, C)
    dw, dwp = row(weight, C), row(post_weight, C)
    need = attn_jvp_adaln_bwd_workspace_bytes(B, L, C)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    elif workspace.device != x.device:
        raise ValueError(f"workspace must be on {x.device}")
    with torch.cuda.device(x.device):
        _raise(attn_jvp_adaln_bwd(a, dx_new, dy, dx, dh, dgate, dscale, dshift, dw, dwp, workspace,
                                  workspace.numel() * workspace.element_size(), torch.cuda.current_stream().cuda_stream))
    return AdaLNGrads(dx, dh, dgate, dscale, dshift, dw, dwp)
