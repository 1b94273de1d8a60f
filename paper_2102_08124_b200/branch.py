"""Autograd forms of the residual branch's operators: dropout from a counter-based generator and the root-mean-square norm of a residual sum.

Random numbers hang on (seed, offset): give every use its own offset, and every step too.  In a captured graph pass `offset_dev` (int64[1] on the
device, added to the offset when the kernels run) and raise it once a step, behind the backward pass."""
from __future__ import annotations

from . import binding as tm
from . import binding_branch as bb

_functions = None


def _rows(t):
    """As a matrix whose rows lie apart from each other, copied if need be (the gradient of a sum is an expanded scalar or row)."""
    t = t.reshape(t.shape[:-1].numel(), t.shape[-1])                     # not -1, which tensors without columns do not tell
    apart = (t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])
    return t if apart else t.contiguous()


def _make():
    import torch
    from torch.autograd.function import once_differentiable              # second derivatives are refused, not left out

    class Dropout(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, offset_dev, p, seed, offset):
            ctx.random = (p, seed, offset)
            ctx.save_for_backward(offset_dev)
            x2, y = _rows(x), torch.empty(x.shape, dtype=x.dtype, device=x.device)
            bb.tm_dropout(x2, p, seed, offset, residual=None if residual is None else _rows(residual), y=y.view(x2.shape), offset_dev=offset_dev)
            return y

        @staticmethod
        def backward(ctx, dy):                              # linear in x: its gradient is the operator itself
            (offset_dev,) = ctx.saved_tensors
            dx = Dropout.apply(dy, None, offset_dev, *ctx.random) if ctx.needs_input_grad[0] else None
            return dx, dy if ctx.needs_input_grad[1] else None, None, None, None, None

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, offset_dev, eps, p, seed, offset):
            x2 = _rows(x)
            # outputs of x's shape, of which the kernel gets views: a view itself could not be written to in place
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            h = None if residual is None and p == 0 else torch.empty_like(y)
            _, _, rstd = bb.tm_rms_norm(x2, weight, eps, residual=None if residual is None else _rows(residual), p=p, seed=seed, offset=offset,
                                        offset_dev=offset_dev, y=y.view(x2.shape), sum_out=None if h is None else h.view(x2.shape))
            ctx.save_for_backward(x2 if h is None else h, rstd, weight, offset_dev)
            ctx.random, ctx.shape = (p, seed, offset), x.shape
            ctx.set_materialize_grads(False)
            # where the sum is x itself, its other uses reach x by their own way
            return y, h

        @staticmethod
        @once_differentiable
        def backward(ctx, dy, dsum):
            h, rstd, weight, offset_dev = ctx.saved_tensors
            p, seed, offset = ctx.random
            need = ctx.needs_input_grad
            if dy is None and dsum is None:
                return (None,) * 8
            h = _rows(h)
            if dy is None:                                  # only the sum was used
                dy = torch.zeros_like(h)
            dh, dx, dw = bb.tm_rms_norm_backward(_rows(dy), h, rstd, weight, dsum=None if dsum is None else _rows(dsum), p=p, seed=seed, offset=offset,
                                                 offset_dev=offset_dev, want_dh=need[1], want_weight=need[2])
            # with p = 0 both are one tensor, and stay one: autograd copies a tensor that it gets twice, but not two views of it
            one = dh is dx
            dx = dx.view(ctx.shape)
            dh = dx if one else dh.view(ctx.shape) if need[1] else None
            return (dx if need[0] else None, dh if need[1] else None, dw) + (None,) * 5

    return Dropout, Norm


def _get():
    global _functions
    if _functions is None:
        _functions = _make()
    return _functions


def _same(x, residual):
    if residual is not None and residual.shape != x.shape:               # rows of other shapes could still be as many
        raise tm.TmError(2, "residual must have the shape of x")


def dropout(x, p: float, seed: int, offset: int = 0, residual=None, offset_dev=None):
    """Differentiable dropout of x [..., cols], plus residual where given; the mask is worked out again for the gradient."""
    _same(x, residual)
    return _get()[0].apply(x, residual, offset_dev, p, seed, offset)


def rms_norm(x, weight=None, eps: float = 1e-5, residual=None, p: float = 0.0, seed: int = 0, offset: int = 0, offset_dev=None):
    """Differentiable root-mean-square norm over the last dimension of dropout(x) (+ residual).  Returns (y, the sum); the sum is x without
    a residual and with p = 0."""
    _same(x, residual)
    y, h = _get()[1].apply(x, residual, weight, offset_dev, eps, p, seed, offset)
    return y, x if h is None else h
