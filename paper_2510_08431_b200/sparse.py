"""Attention over selected key blocks (``attn_jvp_block_select``, ``attn_jvp_sparse_*``): binding and tensor checks.

Every block of 128 queries attends only to the blocks of 128 keys kept for it: by ``block_select`` (the topk largest dot
products of block means) or by a caller's mask (``block_selection``).  ``sparse_attention_jvp`` is ``attention_jvp`` over
such a selection, ``sparse_attention_backward`` its gradients.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import attn_jvp as _binding
from .attn_jvp import _ptr

SELECT_BLOCK = 128


def attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D) -> int:
    return int(_binding.load().attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D))


def attn_jvp_block_select(q, k, B, H, Lq, Lk, D, topk, mask, index, tiles, workspace, workspace_bytes, cuda_stream) -> int:
    return _binding.load().attn_jvp_block_select(_ptr(q), _ptr(k), B, H, Lq, Lk, D, int(topk), _ptr(mask), _ptr(index),
                                                 _ptr(tiles), _ptr(workspace), int(workspace_bytes), _ptr(cuda_stream))


def attn_jvp_block_lists(mask, B, H, Lq, Lk, index, tiles, order, cuda_stream) -> int:
    return _binding.load().attn_jvp_block_lists(_ptr(mask), B, H, Lq, Lk, _ptr(index), _ptr(tiles), _ptr(order), _ptr(cuda_stream))


def attn_jvp_sparse_fwd(q, k, v, tq, tk, tv, index, tiles, order, o, to, lse, mu, B, H, Lq, Lk, D, scale, flags, cuda_stream) -> int:
    return _binding.load().attn_jvp_sparse_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(tq), _ptr(tk), _ptr(tv), _ptr(index),
                                                _ptr(tiles), _ptr(order), _ptr(o), _ptr(to), _ptr(lse), _ptr(mu), B, H, Lq, Lk, D,
                                                float(scale), int(flags), _ptr(cuda_stream))


def attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D) -> int:
    return int(_binding.load().attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D))


def attn_jvp_sparse_bwd(d_o, q, k, v, o, lse, mask, index, tiles, order, dq, dk, dv, B, H, Lq, Lk, D, scale, workspace,
                        workspace_bytes, cuda_stream) -> int:
    return _binding.load().attn_jvp_sparse_bwd(_ptr(d_o), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(mask),
                                               _ptr(index), _ptr(tiles), _ptr(order), _ptr(dq), _ptr(dk), _ptr(dv), B, H, Lq, Lk, D,
                                               float(scale), _ptr(workspace), int(workspace_bytes), _ptr(cuda_stream))


class BlockSelection(NamedTuple):
    """Which key blocks each query block attends to.  Made by ``block_select`` or ``block_selection``; immutable: the
    lists are those of the mask, and changing one by hand would leave the others behind."""
    mask: torch.Tensor       # bool [B][H][n_q][n_k]
    index: torch.Tensor      # int32 [B][H][n_q][n_k], ascending, the first entries of a row count
    tiles: torch.Tensor      # int32 [B][H][n_q], 64-key tiles of a row's blocks
    order: Optional[torch.Tensor]    # int32 [B][H][n_q], all rows in the order of their work; None: as they lie
    Lq: int
    Lk: int


def block_select(q, k, topk, workspace=None) -> BlockSelection:
    """For every (batch, head, block of 128 queries) the ``topk`` key blocks whose mean key has the largest dot product with
    the block's mean query (64-bit arithmetic, ties to the lower block, NaN above everything; all of them where there are fewer).

    q: [B][Lq][H][D], k: [B][Lk][H][D], contiguous CUDA bf16, D = 64 or 128.  ``workspace``: a CUDA uint8 tensor of at least
    attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D)."""
    rc, mask, index, tiles = _binding.host().block_select(q, k, topk, workspace)
    if rc:
        _binding._raise(rc)
    return BlockSelection(mask, index, tiles, None, q.shape[1], k.shape[1])


def block_selection(mask, Lq, Lk) -> BlockSelection:
    """The selection of a caller's mask: contiguous CUDA bool [B][H][ceil(Lq / 128)][ceil(Lk / 128)].  The mask is kept, not
    copied: it must not be written to while the selection is in use, the gradients of keys and values read it again."""
    rc, index, tiles, order = _binding.host().block_lists(mask, Lq, Lk)
    if rc:
        _binding._raise(rc)
    return BlockSelection(mask, index, tiles, order, Lq, Lk)


def _selection(sel) -> BlockSelection:
    if not isinstance(sel, BlockSelection):
        raise ValueError("the selection must come from block_select or block_selection")
    return sel


def sparse_attention_jvp(q, k, v, selection, tq=None, tk=None, tv=None, scale=None, fwd_only=False, out=None, return_mu=False):
    """``attention_jvp`` over the kept key blocks: (o, to, lse) or (o, to, lse, mu), on torch's current stream.

    Arguments as ``attention_jvp``; ``selection``: a ``BlockSelection`` for these sizes.  Rows of a query block without any
    key: o = to = 0, lse = -inf.  The selection does not move with the tangents."""
    rc, o, to, lse, mu = _binding.host().sparse_fwd(q, k, v, *_selection(selection), tq, tk, tv, scale, bool(fwd_only),
                                                    bool(return_mu), *(out or (None, None, None)))
    if rc:
        _binding._raise(rc)
    return (o, to, lse, mu) if return_mu else (o, to, lse)


def sparse_attention_backward(d_o, q, k, v, o, lse, selection, scale=None, workspace=None):
    """(dq, dk, dv) of ``sparse_attention_jvp(..., fwd_only=True)`` for the gradient ``d_o`` of its o.

    ``o``, ``lse``: what that call returned.  ``workspace``: a CUDA uint8 tensor of at least
    attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D), 256-byte aligned."""
    rc, dq, dk, dv = _binding.host().sparse_bwd(d_o, q, k, v, o, lse, *_selection(selection), scale, workspace)
    if rc:
        _binding._raise(rc)
    return dq, dk, dv
