"""The differentiable operators of `train_ops` as autograd functions: what a model calls.  They can be differentiated once: a
second derivative through them raises."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import train_ops


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t itself where the kernels can read it as rows of its last dimension, otherwise a copy."""
    if t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]):
        return t
    return t.contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        x = _rows(x)
        weight, bias = (None if t is None else t.contiguous() for t in (weight, bias))
        y, stats = train_ops.layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, stats)
        ctx.bias_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        need = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dw, db = train_ops.layer_norm_backward(_rows(dy), x, weight, stats, need_params=need)
        return (dx if ctx.needs_input_grad[0] else None, dw.to(weight.dtype) if ctx.needs_input_grad[1] else None,
                db.to(ctx.bias_dtype) if ctx.needs_input_grad[2] else None, None)


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, top, scale):
        logits, ids = _rows(logits), ids.contiguous()
        r = train_ops.token_logprobs(logits, ids, top=top, scale=scale)
        logp, entropy, lse = (t.clone() for t in r.stats)
        top_idx = r.top_idx if top else torch.empty((logits.shape[0], 0), dtype=torch.int32, device=logits.device)
        top_logp = r.top_logp if top else torch.empty((logits.shape[0], 0), device=logits.device)
        ctx.mark_non_differentiable(lse, top_idx)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, ids, r.stats, top_idx)
        ctx.scale = scale
        return logp, entropy, lse, top_idx, top_logp

    @staticmethod
    @once_differentiable
    def backward(ctx, d_logp, d_entropy, _lse, _idx, d_top):
        logits, ids, stats, top_idx = ctx.saved_tensors
        whole = lambda t: None if t is None else t.contiguous()  # noqa: E731
        top = d_top is not None and top_idx.shape[1] > 0
        return train_ops.token_logprobs_backward(
            logits, ids, stats[2], whole(d_logp), entropy=stats[1], d_entropy=whole(d_entropy),
            top_idx=top_idx if top else None, d_top=whole(d_top) if top else None, scale=ctx.scale), None, None, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5) -> torch.Tensor:
    """`train_ops.layer_norm` with gradients for x, weight and bias.  What does not lie in rows is copied first."""
    return _LayerNorm.apply(x, weight, bias, eps)


def token_logprobs(logits, ids, top: int = 0, scale: float = 1.0):
    """(logp, entropy, lse, top_idx, top_logp) of `train_ops.token_logprobs`.  logp, entropy and top_logp have gradients; lse, which
    the backward pass reads, has none.  Logits that do not lie in rows are copied first."""
    return _TokenLogprobs.apply(logits, ids, top, scale)
