"""Layer-level front end: the attention core, dense or over selected key blocks, and the step between two branches of a
DiT block, each of which runs either as a plain call or in JVP mode.

The paper restructures every network layer so that one call can carry primals alone or (primal, tangent)
pairs, selected by a ``withT`` keyword (Appendix C.2, "Network Restructuring"); all layers use PyTorch's
forward-mode operator for the JVP branch except the attention core, which calls the fused kernel
(Appendix C.1).  Here the attention core for [B][L][H][D] bf16 tensors and the norms around it run in the CUDA library
in both modes; the plain calls of the layers below the dense core are differentiable (once).  Calls with ``withT`` and the
dense core's plain call are not: their results carry no autograd graph, also where the arguments require grad.
All passes can be captured into a CUDA graph; as with any layer, no autograd graph made outside the capture may then be alive
for the same leaf tensors (the layers themselves keep none).
"""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import adaln as _adaln
from . import attn_jvp as _binding
from . import sparse as _sparse

TensorWithT = Tuple[torch.Tensor, torch.Tensor]   # (primal, tangent)


class AttentionCoreJVP(torch.nn.Module):
    """softmax(s q k^T) v with an optional tangent channel.

    ``forward(q, k, v)`` returns O.  ``forward(q, k, v, withT=True)`` takes q as a (primal, tangent) pair and
    k, v either as pairs (self-attention: their tangents matter) or as plain tensors (cross-attention on a
    context that does not depend on the differentiated input, so tK = tV = 0), and returns (O, tO).
    The log-sum-exp of the last call is kept in ``self.last_lse`` (and mu, the tangent of the LSE, in
    ``self.last_mu`` when ``keep_mu`` is set).
    """

    def __init__(self, scale: Optional[float] = None, keep_mu: bool = False):
        super().__init__()
        self.scale = scale
        self.keep_mu = keep_mu
        self.last_lse = None
        self.last_mu = None

    def forward(self, q, k, v, withT: bool = False):
        if withT:
            return self._forward_jvp(q, k, v)
        return self._forward(q, k, v)

    def _forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
        o, _, lse = _binding.attention_jvp(q, k, v, scale=self.scale, fwd_only=True)
        self.last_lse, self.last_mu = lse, None
        return o

    def _forward_jvp(self, q: TensorWithT, k: Union[TensorWithT, torch.Tensor],
                     v: Union[TensorWithT, torch.Tensor]) -> TensorWithT:
        qp, qt = q
        k_pair, v_pair = isinstance(k, (tuple, list)), isinstance(v, (tuple, list))
        if k_pair != v_pair:
            raise ValueError("k and v must both carry tangents (self-attention) or both be constant (context)")
        if k_pair:
            (kp, kt), (vp, vt) = k, v
        else:
            kp, kt, vp, vt = k, None, v, None
        res = _binding.attention_jvp(qp, kp, vp, qt.detach(), None if kt is None else kt.detach(),
                                     None if vt is None else vt.detach(), scale=self.scale,
                                     return_mu=self.keep_mu)
        self.last_lse = res[2]
        self.last_mu = res[3] if self.keep_mu else None
        return res[0], res[1]


def _pair(v):
    """(primal, tangent) of a value that may carry a tangent."""
    return v if isinstance(v, (tuple, list)) else (v, None)


class _FirstOrder(torch.autograd.Function):
    """A gradient as a function of what it was computed from, whose own gradient does not exist."""

    @staticmethod
    def forward(ctx, grad, *inputs):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("second derivatives of this layer are not available")


def _first_order(grads, *inputs):
    """Under create_graph a gradient's own gradient must be an error: left as a constant, it would silently count as zero."""
    if not torch.is_grad_enabled():
        return grads
    return tuple(None if g is None else _FirstOrder.apply(g, *inputs) for g in grads)


class _AdaLN(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, h, gate, scale, shift, weight, post_weight, kinds):
        ctx.set_materialize_grads(False)
        ctx.kinds = kinds
        ctx.save_for_backward(x, h, gate, scale, shift, weight, post_weight)
        xn, y, _, _ = _adaln.adaln_jvp(x, h, gate, scale, shift, weight, post_weight, **kinds)
        return (x.view_as(x) if h is None else xn), y

    @staticmethod
    def backward(ctx, dxn, dy):
        x, h, gate, scale, shift, weight, post_weight = ctx.saved_tensors
        if dxn is None and dy is None:
            return (None,) * 8
        g = _adaln.adaln_backward(None if dxn is None else dxn.contiguous(), None if dy is None else dy.contiguous(), x, h, gate,
                                  scale, shift, weight, post_weight, **ctx.kinds)
        return (*_first_order(g, dxn, dy, *ctx.saved_tensors), None)


class AdaLNJVP(torch.nn.Module):
    """Gate + residual + norm + modulation between two branches of a DiT block (``adaln_jvp``), with an optional tangent
    channel and, without it, autograd.

    ``forward(x, h, gate, scale, shift)`` returns (x', y); h and the modulation may be None.  ``forward(..., withT=True)``
    takes x and h as (primal, tangent) pairs and gate, scale, shift as pairs or as plain tensors (constant), and returns the
    pairs (x', tx') and (y, ty), without an autograd graph.  ``affine`` / ``post_affine`` give the norms learnt fp32 weights (constants of the tangents:
    the JVP runs on the frozen network).
    """

    def __init__(self, dim: int, norm: Optional[str] = "layer", post_norm: Optional[str] = None, eps: float = 1e-6,
                 affine: bool = False, post_affine: bool = False):
        super().__init__()
        self.kinds = dict(norm=norm, post_norm=post_norm, eps=eps)
        self.weight = torch.nn.Parameter(torch.ones(dim)) if affine else None
        self.post_weight = torch.nn.Parameter(torch.ones(dim)) if post_affine else None

    def forward(self, x, h=None, gate=None, scale=None, shift=None, withT: bool = False):
        # (a call without a branch has nothing for the post norm to act on)
        kinds = self.kinds if (_pair(h)[0] if withT else h) is not None else dict(self.kinds, post_norm=None)
        if not withT:
            return _AdaLN.apply(x, h, gate, scale, shift, self.weight, None if h is None else self.post_weight, kinds)
        (x, tx), (h, th) = _pair(x), _pair(h)
        (gate, tgate), (scale, tscale), (shift, tshift) = _pair(gate), _pair(scale), _pair(shift)
        if tx is None or (h is not None and th is None):
            raise ValueError("withT: x and h must carry tangents")
        w = None if self.weight is None else self.weight.detach()
        wp = None if self.post_weight is None or h is None else self.post_weight.detach()
        xn, y, txn, ty = _adaln.adaln_jvp(x, h, gate, scale, shift, w, wp, **kinds, tx=tx.detach(),
                                          th=None if th is None else th.detach(), tgate=tgate, tscale=tscale, tshift=tshift)
        return (xn, txn), (y, ty)


class _SparseAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, selection, scale):
        o, _, lse = _sparse.sparse_attention_jvp(q, k, v, selection, scale=scale, fwd_only=True)
        ctx.lengths, ctx.scale = selection[4:], scale
        ctx.save_for_backward(q, k, v, o, lse, *selection[:4])      # (a mask that is written to meanwhile is an error)
        ctx.mark_non_differentiable(lse)
        return o, lse

    @staticmethod
    def backward(ctx, d_o, _):
        q, k, v, o, lse, *lists = ctx.saved_tensors
        selection = _sparse.BlockSelection(*lists, *ctx.lengths)
        grads = _sparse.sparse_attention_backward(d_o.contiguous(), q, k, v, o, lse, selection, scale=ctx.scale)
        return (*_first_order(grads, d_o, q, k, v), None, None)


class SparseAttentionCoreJVP(torch.nn.Module):
    """``AttentionCoreJVP`` over selected key blocks: every block of 128 queries attends to the ``topk`` blocks of 128 keys
    whose mean key fits its mean query best, or to those of a ``selection`` that the caller passes.

    Plain calls are differentiable (the selection is a constant); ``withT=True`` takes and returns pairs as
    ``AttentionCoreJVP`` does, without an autograd graph.  The selection, log-sum-exp and (``keep_mu``) its tangent of the last call are kept in
    ``last_selection``, ``last_lse`` and ``last_mu``.
    """

    def __init__(self, topk: int, scale: Optional[float] = None, keep_mu: bool = False):
        super().__init__()
        self.topk, self.scale, self.keep_mu = topk, scale, keep_mu
        self.last_selection = self.last_lse = self.last_mu = None

    def forward(self, q, k, v, withT: bool = False, selection=None):
        if withT:
            (q, tq), (k, tk), (v, tv) = _pair(q), _pair(k), _pair(v)
            if (tk is None) != (tv is None):
                raise ValueError("k and v must both carry tangents (self-attention) or both be constant (context)")
            if tq is None:
                raise ValueError("withT: q must carry a tangent")
        if selection is None:
            selection = _sparse.block_select(q.detach(), k.detach(), self.topk)
        self.last_selection, self.last_mu = selection, None
        if not withT:
            o, self.last_lse = _SparseAttention.apply(q, k, v, selection, self.scale)
            return o
        res = _sparse.sparse_attention_jvp(q, k, v, selection, tq.detach(), None if tk is None else tk.detach(),
                                           None if tv is None else tv.detach(), scale=self.scale, return_mu=self.keep_mu)
        self.last_lse = res[2]
        self.last_mu = res[3] if self.keep_mu else None
        return res[0], res[1]
