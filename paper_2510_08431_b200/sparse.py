"""Attention over selected key blocks (``attn_jvp_block_select``, ``attn_jvp_sparse_*``): binding and tensor checks.

Every block of 128 queries attends only to the blocks of 128 keys kept for it: by ``block_select`` (the topk largest dot
products of block means) or by a caller's mask (``block_selection``).  ``sparse_attention_jvp`` is ``attention_jvp`` over
such a selection, ``sparse_attention_backward`` its gradients.
"""
from __future__ import annotations

import math
from typing import NamedTuple

import torch

from . import attn_jvp as _binding
from .attn_jvp import FWD_ONLY, KV_TANGENT_FREE, _call_on, _ptr

SELECT_BLOCK = 128


def attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D) -> int:
    return int(_binding.load().attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D))


def attn_jvp_block_select(q, k, B, H, Lq, Lk, D, topk, mask, index, tiles, workspace, workspace_bytes, cuda_stream) -> int:
    return (_binding.load().attn_jvp_block_select(_ptr(q), _ptr(k), B, H, Lq, Lk, D, int(topk), _ptr(mask), _ptr(index),
                                                     _ptr(tiles), _ptr(workspace), int(workspace_bytes), _ptr(cuda_stream)))


def attn_jvp_block_lists(mask, B, H, Lq, Lk, index, tiles, cuda_stream) -> int:
    return int(_binding.load().attn_jvp_block_lists(_ptr(mask), B, H, Lq, Lk, _ptr(index), _ptr(tiles), _ptr(cuda_stream)))


def attn_jvp_sparse_fwd(q, k, v, tq, tk, tv, index, tiles, o, to, lse, mu, B, H, Lq, Lk, D, scale, flags, cuda_stream) -> int:
    return (_binding.load().attn_jvp_sparse_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(tq), _ptr(tk), _ptr(tv), _ptr(index),
                                                   _ptr(tiles), _ptr(o), _ptr(to), _ptr(lse), _ptr(mu), B, H, Lq, Lk, D,
                                                   float(scale), int(flags), _ptr(cuda_stream)))


def attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D) -> int:
    return int(_binding.load().attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D))


def attn_jvp_sparse_bwd(d_o, q, k, v, o, lse, mask, index, tiles, dq, dk, dv, B, H, Lq, Lk, D, scale, workspace,
                        workspace_bytes, cuda_stream) -> int:
    return (_binding.load().attn_jvp_sparse_bwd(_ptr(d_o), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(mask),
                                                   _ptr(index), _ptr(tiles), _ptr(dq), _ptr(dk), _ptr(dv), B, H, Lq, Lk, D,
                                                   float(scale), _ptr(workspace), int(workspace_bytes), _ptr(cuda_stream)))


def _check(t, name, shape, device):
    if t.dtype is not torch.bfloat16 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous bf16 tensor of shape {tuple(shape)} on {device}")


def _check_qkv(q, k, v):
    """Sizes of the call; q, k, v (or None) checked."""
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be CUDA tensors [B][L][H][D]")
    B, Lq, H, D = q.shape
    dev, kv = q.device, (B, k.shape[1], H, D)
    _check(q, "q", q.shape, dev)
    _check(k, "k", kv, dev)
    if v is not None:
        _check(v, "v", kv, dev)
    return B, H, Lq, kv[1], D


class BlockSelection(NamedTuple):
    """Which key blocks each query block attends to.  Made by ``block_select`` or ``block_selection``; immutable: the
    lists are those of the mask, and changing one by hand would leave the others behind."""
    mask: torch.Tensor       # bool [B][H][n_q][n_k]
    index: torch.Tensor      # int32 [B][H][n_q][n_k], ascending, the first entries of a row count
    tiles: torch.Tensor      # int32 [B][H][n_q], 64-key tiles of a row's blocks
    Lq: int
    Lk: int


def _blocks(L):
    return -(-L // SELECT_BLOCK)


def _lists(t, B, H, n_q, n_k):
    return t.new_empty((B, H, n_q, n_k), dtype=torch.int32), t.new_empty((B, H, n_q), dtype=torch.int32)


def block_select(q, k, topk, workspace=None) -> BlockSelection:
    """For every (batch, head, block of 128 queries) the ``topk`` key blocks whose mean key has the largest dot product with
    the block's mean query (64-bit arithmetic, ties to the lower block; all of them where there are fewer).

    q: [B][Lq][H][D], k: [B][Lk][H][D], contiguous CUDA bf16, D = 64 or 128.  ``workspace``: a CUDA uint8 tensor of at least
    attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D)."""
    B, H, Lq, Lk, D = _check_qkv(q, k, None)
    need = attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D)
    if workspace is None:
        workspace, size = q.new_empty(need, dtype=torch.uint8), need
    elif workspace.device != q.device:
        raise ValueError(f"workspace must be on {q.device}")
    else:
        size = workspace.numel() * workspace.element_size()
    n_q, n_k = _blocks(Lq), _blocks(Lk)
    mask = q.new_empty((B, H, n_q, n_k), dtype=torch.bool)
    index, tiles = _lists(q, B, H, n_q, n_k)
    _call_on(q.device, attn_jvp_block_select, q, k, B, H, Lq, Lk, D, topk, mask, index, tiles, workspace, size)
    return BlockSelection(mask, index, tiles, Lq, Lk)


def block_selection(mask, Lq, Lk) -> BlockSelection:
    """The selection of a caller's mask: contiguous CUDA bool [B][H][ceil(Lq / 128)][ceil(Lk / 128)].  The mask is kept, not
    copied: later writes to it do not reach the lists."""
    if not mask.is_cuda or mask.dtype != torch.bool or mask.dim() != 4 or not mask.is_contiguous():
        raise ValueError("mask must be a contiguous CUDA bool tensor [B][H][n_q][n_k]")
    B, H = mask.shape[:2]
    if tuple(mask.shape[2:]) != (_blocks(Lq), _blocks(Lk)):
        raise ValueError(f"mask must have {_blocks(Lq)} x {_blocks(Lk)} blocks for {Lq} queries and {Lk} keys")
    index, tiles = _lists(mask, B, H, _blocks(Lq), _blocks(Lk))
    _call_on(mask.device, attn_jvp_block_lists, mask, B, H, Lq, Lk, index, tiles)
    return BlockSelection(mask, index, tiles, Lq, Lk)


def _check_selection(sel, B, H, Lq, Lk, device):
    if not isinstance(sel, BlockSelection):
        raise ValueError("the selection must come from block_select or block_selection")
    if sel.Lq != Lq or sel.Lk != Lk or sel.mask.shape[:2] != (B, H) or sel.mask.device != device:
        raise ValueError(f"the selection is for other sizes or another device than q and k (B={B}, H={H}, Lq={Lq}, Lk={Lk})")


def sparse_attention_jvp(q, k, v, selection, tq=None, tk=None, tv=None, scale=None, fwd_only=False, out=None, return_mu=False):
    """``attention_jvp`` over the kept key blocks: (o, to, lse) or (o, to, lse, mu), on torch's current stream.

    Arguments as ``attention_jvp``; ``selection``: a ``BlockSelection`` for these sizes.  Rows of a query block without any
    key: o = to = 0, lse = -inf.  The selection does not move with the tangents."""
    B, H, Lq, Lk, D = _check_qkv(q, k, v)
    dev = q.device
    _check_selection(selection, B, H, Lq, Lk, dev)
    flags = 0
    if fwd_only:
        flags = FWD_ONLY
        tq = tk = tv = None
    else:
        if tq is None:
            raise ValueError("tq is required unless fwd_only")
        _check(tq, "tq", q.shape, dev)
        if tk is None and tv is None:
            flags = KV_TANGENT_FREE
        elif tk is None or tv is None:
            raise ValueError("tk and tv must both be given or both be None")
        else:
            _check(tk, "tk", k.shape, dev)
            _check(tv, "tv", k.shape, dev)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        o = torch.empty_like(q)
        to = None if fwd_only else torch.empty_like(q)
        lse = q.new_empty((B, H, Lq), dtype=torch.float32)
    else:
        o, to, lse = out
    mu = q.new_empty((B, H, Lq), dtype=torch.float32) if return_mu else None
    _call_on(dev, attn_jvp_sparse_fwd, q, k, v, tq, tk, tv, selection.index, selection.tiles, o, to, lse, mu, B, H, Lq, Lk, D, scale,
             flags)
    return (o, to, lse, mu) if return_mu else (o, to, lse)


def sparse_attention_backward(d_o, q, k, v, o, lse, selection, scale=None, workspace=None):
    """(dq, dk, dv) of ``sparse_attention_jvp(..., fwd_only=True)`` for the gradient ``d_o`` of its o.

    ``o``, ``lse``: what that call returned.  ``workspace``: a CUDA uint8 tensor of at least
    attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D), 256-byte aligned."""
    B, H, Lq, Lk, D = _check_qkv(q, k, v)
    dev = q.device
    _check(o, "o", q.shape, dev)
    _check(d_o, "d_o", q.shape, dev)
    if lse.dtype is not torch.float32 or lse.device != dev or lse.shape != (B, H, Lq) or not lse.is_contiguous():
        raise ValueError(f"lse must be a contiguous fp32 tensor of shape {(B, H, Lq)} on {dev}")
    _check_selection(selection, B, H, Lq, Lk, dev)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    need = attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D)
    if workspace is None:
        workspace, size = q.new_empty(need, dtype=torch.uint8), need
    elif workspace.device != dev:
        raise ValueError(f"workspace must be on {dev}")
    else:
        size = workspace.numel() * workspace.element_size()
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    _call_on(dev, attn_jvp_sparse_bwd, d_o, q, k, v, o, lse, selection.mask, selection.index, selection.tiles, dq, dk, dv, B, H, Lq,
             Lk, D, scale, workspace, size)
    return dq, dk, dv
