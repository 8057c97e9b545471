"""The step between two branches of a DiT block: gate + residual + norm + modulation, fused (``attn_jvp_adaln_*``).

    u  = post_weight . post_norm(h),   x' = x + gate . u,   y = weight . norm(x') (1 + scale) + shift

A block calls it once per branch: y of one call is the input of the next attention or MLP branch, whose output is the
next call's h.  Forward, forward with tangents (the JVP mode of the generator step) and backward (the student step).
Argument checks and allocation happen in the host binding, the arithmetic in the CUDA library; there is no CPU path.
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


def _kinds(norm, post_norm):
    try:
        return NORMS[norm], NORMS[post_norm]
    except (KeyError, TypeError):
        raise ValueError(f"norm and post_norm are one of {list(NORMS)}") from None


def adaln_jvp(x, h=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, norm="layer", post_norm=None,
              eps=1e-6, tx=None, th=None, tgate=None, tscale=None, tshift=None):
    """x' = x + gate . post_weight . post_norm(h) and y = weight . norm(x') (1 + scale) + shift, with tangents if given.

    x: [B][L][C] CUDA bf16 or fp32; h: bf16 [B][L][C] or None (x' is x itself then); gate, scale, shift: fp32 [B][C] with
    any row stride (a slice of a [B][6][C] modulation, a broadcast row) or None; weight, post_weight: fp32 [C] or None;
    norm, post_norm: "layer", "rms" or None (norm=None: y is None).  C: a multiple of 8 up to 8192.  ``tx`` (type of x),
    ``th`` (bf16) and optionally tgate, tscale, tshift select the JVP mode.
    Returns (x', y, tx', ty); x', tx' have the type of x, y, ty are bf16; the tangents are None without ``tx``.
    """
    kind, post_kind = _kinds(norm, post_norm)
    rc, xn, y, txn, ty = _binding.host().adaln_fwd(x, h, gate, scale, shift, weight, post_weight, kind, post_kind, eps, tx, th,
                                                   tgate, tscale, tshift)
    if rc:
        _binding._raise(rc)
    return (x, y, tx, ty) if h is None else (xn, y, txn, ty)


def adaln_backward(dx_new, dy, x, h=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, norm="layer",
                   post_norm=None, eps=1e-6, workspace=None) -> AdaLNGrads:
    """Gradients of ``adaln_jvp`` for dx' (type of x, or None: 0) and dy (bf16, or None: 0).

    The forward's inputs are passed again; its statistics are recomputed in the same pass.  Gradients of x have the type
    of x, of h bf16, of the modulation fp32 [B][C] (one row per sample also where the input's rows were shared), of the
    weights fp32 [C].  ``workspace``: a CUDA uint8 tensor of at least attn_jvp_adaln_bwd_workspace_bytes(B, L, C).
    """
    kind, post_kind = _kinds(norm, post_norm)
    rc, *grads = _binding.host().adaln_bwd(dx_new, dy, x, h, gate, scale, shift, weight, post_weight, kind, post_kind, eps, workspace)
    if rc:
        _binding._raise(rc)
    return AdaLNGrads(*grads)
