"""Dense attention with a causal mask, key lengths, shared key heads and strided inputs (``attn_jvp_attention_*``): raw calls, and the
gradients of ``attention_jvp``'s plain forward, masked or not.
"""
from __future__ import annotations

import ctypes

from . import attn_jvp as _binding


class AttentionArgs(ctypes.Structure):
    """attn_jvp_attention_t of include/attn_jvp.h."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "tq", "tk", "tv", "k_lengths")]
                + [(n + "_stride", ctypes.c_longlong * 3) for n in ("q", "k", "v")]
                + [(n, ctypes.c_int) for n in ("B", "H", "Hk", "Lq", "Lk", "D", "causal")] + [("scale", ctypes.c_float)])


def attn_jvp_attention_fwd(args: AttentionArgs, o, to, lse, mu, flags, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_attention_fwd(ctypes.byref(args), p(o), p(to), p(lse), p(mu), int(flags), p(cuda_stream))


def attn_jvp_attention_bwd_workspace_bytes(B, H, Hk, Lq, Lk, D) -> int:
    return int(_binding.load().attn_jvp_attention_bwd_workspace_bytes(int(B), int(H), int(Hk), int(Lq), int(Lk), int(D)))


def attn_jvp_attention_bwd(args: AttentionArgs, d_o, o, lse, dq, dk, dv, workspace, workspace_bytes, cuda_stream) -> int:
    p = _binding._ptr
    return _binding.load().attn_jvp_attention_bwd(ctypes.byref(args), p(d_o), p(o), p(lse), p(dq), p(dk), p(dv), p(workspace),
                                                  int(workspace_bytes), p(cuda_stream))


def attention_backward(d_o, q, k, v, o, lse, scale=None, causal=False, k_lengths=None, workspace=None):
    """(dq, dk, dv) of ``attention_jvp(q, k, v, scale=scale, fwd_only=True, causal=causal, k_lengths=k_lengths)`` for the gradient ``d_o``
    of its o.  The probabilities are recomputed from ``lse``; gradients of shared key heads are sums over the heads that share them.

    ``o``, ``lse``: what that call returned; d_o, o contiguous bf16 [B][Lq][H][D].  Gradients are contiguous bf16 and do not change from run to run.
    ``workspace``: a CUDA uint8 tensor of at least attn_jvp_attention_bwd_workspace_bytes(B, H, Hk, Lq, Lk, D), 256-byte aligned."""
    rc, dq, dk, dv = _binding.host().attention_bwd(d_o, q, k, v, scale, bool(causal), k_lengths, o, lse, workspace)
    if rc:
        _binding._raise(rc)
    return dq, dk, dv
