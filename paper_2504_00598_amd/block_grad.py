"""The decoder-block operators as recorded functions.

`block` calls these where gradients are recorded and one of the inputs requires one: the forward call and its
`*_bwd`, tied together for backward().  A gradient that is asked for reaches q, k, wq and wk; logits; x, w1, w2
and weight.  It has none of its own (a second derivative is refused).  Backward runs on the stream of the forward
call, as torch does for its own functions.  The recorded program may hold the last reference to an input and drops it
while that stream still reads it, so inputs of a call that names a stream are marked as used on it.
"""
from __future__ import annotations

import torch
from torch.autograd import Function
from torch.autograd.function import once_differentiable

from . import block


def _last(t):
    """t with its last dimension contiguous, which a broadcast gradient has not."""
    return t if t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


class QkNormRope(Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps, interleaved, axes=None):
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        ctx.how = {"eps": eps, "interleaved": interleaved, "axes": None if axes is None else tuple(axes)}
        return block.qk_norm_rope(q, k, wq, wk, cos, sin, positions, **ctx.how)

    @staticmethod
    @once_differentiable
    def backward(ctx, dyq, dyk):
        wq, wk = ctx.saved_tensors[2:4]
        dq, dk, dwq, dwk = block.qk_norm_rope_bwd(_last(dyq), _last(dyk), *ctx.saved_tensors, **ctx.how)
        return (dq, dk, None if wq is None else dwq.to(wq.dtype), None if wk is None else dwk.to(wk.dtype),
                None, None, None, None, None, None)


class Route(Function):
    @staticmethod
    def forward(ctx, logits, k, choice, weights):
        weight, index = block.route(logits, k, **choice, **weights)
        ctx.mark_non_differentiable(index)
        ctx.save_for_backward(logits, index)
        ctx.how = weights
        return weight, index

    @staticmethod
    @once_differentiable
    def backward(ctx, dweight, _):
        return block.route_bwd(dweight, *ctx.saved_tensors, **ctx.how), None, None, None


class Experts(Function):
    @staticmethod
    def forward(ctx, x, w1, w2, weight, plan, ws):
        y, kept = block.experts(x, w1, w2, weight, plan, keep=True, ws=ws)
        ctx.mark_non_differentiable(kept)
        ctx.save_for_backward(x, w1, w2, weight, kept)
        ctx.plan = plan
        return y, kept

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, _):
        *args, kept = ctx.saved_tensors
        # rows that overlap, as a broadcast gradient's, are laid out
        dy = dy if dy.stride(0) >= dy.shape[1] and dy.stride(1) == 1 else dy.contiguous()
        return (*block.experts_bwd(dy, *args, ctx.plan, kept), None, None)


def _used_on(stream, *tensors):
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps, interleaved, stream, axes=None):
    if cos.requires_grad or sin.requires_grad:
        raise ValueError("cos and sin have no gradient")
    _used_on(stream, q, k, wq, wk, cos, sin, positions)
    return QkNormRope.apply(q, k, wq, wk, cos, sin, positions, eps, interleaved, axes)


def route(logits, k, choice, weights, stream):
    _used_on(stream, logits, choice["bias"])
    return Route.apply(logits, k, choice, weights)


def experts(x, w1, w2, weight, plan, keep, ws, stream):
    _used_on(stream, x, w1, w2, weight, plan._buf, ws)
    y, kept = Experts.apply(x, w1, w2, weight, plan, ws)
    return (y, kept) if keep else y
