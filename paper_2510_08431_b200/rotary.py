"""Rotary positions: the table of angles (``attn_jvp_rotary_table``), and the step in front of the attention core that normalises
and rotates the heads of queries and keys (``attn_jvp_qk_rotary_*``): forward, with tangents, gradients.

    u = weight . norm(x) + bias over each head,   y = u with its first R channels turned by pairs

Argument checks and allocation happen in the host binding, the arithmetic in the CUDA library; there is no CPU path.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import attn_jvp as _binding
from .adaln import NORMS

SCALINGS = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}
LAYOUTS = {"interleaved": 0, "half": 1}


class QKRotaryArgs(ctypes.Structure):
    """attn_jvp_qk_rotary_t of include/attn_jvp.h."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "tq", "tk", "q_weight", "k_weight", "q_bias", "k_bias", "table", "index")]
                + [(n + "_stride", ctypes.c_longlong * 3) for n in ("q", "k", "tq", "tk")]
                + [(n, ctypes.c_longlong) for n in ("table_rows", "table_batch", "index_batch")]
                + [(n, ctypes.c_int) for n in ("B", "L", "H", "Hk", "D", "R", "norm", "layout")] + [("eps", ctypes.c_float)])


class QKRotaryGrads(NamedTuple):
    """Gradients of ``qk_rotary_jvp``; None where the input was None (``q`` always has one)."""
    q: torch.Tensor
    k: Optional[torch.Tensor]
    q_weight: Optional[torch.Tensor]
    k_weight: Optional[torch.Tensor]
    q_bias: Optional[torch.Tensor]
    k_bias: Optional[torch.Tensor]


def attn_jvp_rotary_table(positions, pos_type, n, dims, base, scaling, factor, original_length, table, cuda_stream) -> int:
    """Raw call: ``dims``, ``base`` and ``factor`` are sequences of one length, the rest as in include/attn_jvp.h."""
    axes, p = len(dims), _binding._ptr
    return _binding.load().attn_jvp_rotary_table(p(positions), int(pos_type), int(n), axes, (ctypes.c_int * axes)(*dims),
                                                 (ctypes.c_double * axes)(*base), int(scaling), (ctypes.c_double * axes)(*factor),
                                                 float(original_length), p(table), p(cuda_stream))


def attn_jvp_qk_rotary_fwd(args: QKRotaryArgs, q_new, k_new, tq_new, tk_new, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_qk_rotary_fwd(ctypes.byref(args), p(q_new), p(k_new), p(tq_new), p(tk_new), p(cuda_stream))


def attn_jvp_qk_rotary_bwd_workspace_bytes(B, L, H, Hk, D) -> int:
    return int(_binding.load().attn_jvp_qk_rotary_bwd_workspace_bytes(int(B), int(L), int(H), int(Hk), int(D)))


def attn_jvp_qk_rotary_bwd(args: QKRotaryArgs, dq_new, dk_new, dq, dk, dq_weight, dk_weight, dq_bias, dk_bias, workspace,
                           workspace_bytes, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_qk_rotary_bwd(ctypes.byref(args), p(dq_new), p(dk_new), p(dq), p(dk), p(dq_weight), p(dk_weight),
                                                  p(dq_bias), p(dk_bias), p(workspace), int(workspace_bytes), p(cuda_stream))


def _per_axis(v, axes):
    return tuple(v) if isinstance(v, (tuple, list)) else (v,) * axes


def rotary_table(positions, dims, base=10000.0, scaling=None, factor=1.0, original_length=None):
    """(cos, sin) of every position and pair of channels: fp32 [...][R / 2][2], R the sum of ``dims``.

    positions: CUDA int32, int64 or fp32 [...][axes], contiguous, one coordinate per axis of ``dims`` (frame, row, column); with a single axis
    [...], of any shape.  dims: the even number of channels that each axis turns (a number: one axis); the angle of pair i of an axis is position base^(-2 i / d).
    ``base`` and ``factor`` are numbers or one per axis.  ``scaling`` stretches the axes by their factors, for sequences
    beyond those of training: "linear" (angles / factor), "ntk" (base factor^(d / (d - 2))) or "yarn" (slow pairs / factor, fast
    ones kept, by their turns within ``original_length``; entries times 0.1 log(factor) + 1).  Between slow and fast the share ramps over the turns, as
    in the paper; some released models ramp over the pair's index i instead, and their tables differ there.
    """
    dims = _per_axis(dims, 1)
    if scaling not in SCALINGS:
        raise ValueError(f"scaling is one of {list(SCALINGS)}")
    if (scaling == "yarn") != (original_length is not None):
        raise ValueError("original_length belongs to scaling='yarn'")
    if scaling is None and any(f != 1 for f in _per_axis(factor, 1)):
        raise ValueError("factor without scaling")
    rc, table = _binding.host().rotary_table(positions, dims, _per_axis(base, len(dims)), SCALINGS[scaling], _per_axis(factor, len(dims)),
                                             original_length)
    if rc:
        _binding._raise(rc)
    return table


def _kinds(norm, layout):
    try:
        return NORMS[norm], LAYOUTS[layout]
    except (KeyError, TypeError):
        raise ValueError(f"norm is one of {list(NORMS)}, layout one of {list(LAYOUTS)}") from None


def qk_rotary_jvp(q, k, table, index=None, norm=None, layout="interleaved", eps=1e-6, q_weight=None, k_weight=None, q_bias=None,
                  k_bias=None, tq=None, tk=None):
    """Heads of queries and keys normalised (each with its own weights) and rotated, with tangents if given; one launch.

    q: [B][L][H][D], k: [B][L][Hk][D] or None, CUDA bf16, D = 64 or 128, heads contiguous, other strides multiples of 8 (slices of
    a fused projection).  table: fp32 [rows][R / 2][2] or [B][rows][R / 2][2] (``rotary_table``), R a multiple of 8 up to D: the first R channels
    of a head turn.  A token's table row is its place or, with ``index`` (int32 [L] or [B][L]), the index's entry (outside the table: the
    nearest row).  norm: "layer", "rms" or None; weights and biases: fp32 [D] or None.  layout: pairs (2 i, 2 i + 1) for "interleaved", (i, i + R / 2) for
    "half".  ``tq`` and (where k is given) ``tk`` select the JVP mode; table and weights are constants of it.
    Returns (q', k', tq', tk'), contiguous bf16; the tangents are None without ``tq``, k' and tk' without k.
    """
    kind, pairs = _kinds(norm, layout)
    rc, qn, kn, tqn, tkn = _binding.host().qk_rotary_fwd(q, k, table, index, kind, pairs, eps, q_weight, k_weight, q_bias, k_bias, tq, tk)
    if rc:
        _binding._raise(rc)
    return qn, kn, tqn, tkn


def qk_rotary_backward(dq_new, dk_new, q, k, table, index=None, norm=None, layout="interleaved", eps=1e-6, q_weight=None, k_weight=None,
                       q_bias=None, k_bias=None, workspace=None) -> QKRotaryGrads:
    """Gradients of ``qk_rotary_jvp`` for dq' and dk' (contiguous bf16; dk' None exactly where k is).

    The forward's inputs are passed again; its statistics are recomputed in the same pass.  Gradients of q and k are contiguous bf16,
    those of weights and biases fp32 [D].  ``workspace``: a CUDA uint8 tensor of at least attn_jvp_qk_rotary_bwd_workspace_bytes(B, L, H, Hk, D).
    """
    kind, pairs = _kinds(norm, layout)
    rc, *grads = _binding.host().qk_rotary_bwd(dq_new, dk_new, q, k, table, index, kind, pairs, eps, q_weight, k_weight, q_bias, k_bias, workspace)
    if rc:
        _binding._raise(rc)
    return QKRotaryGrads(*grads)
