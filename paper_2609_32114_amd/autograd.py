"""Differentiable forms of the gated linear recurrence and the block norms.

    h, final = glr(x, g, initial_state=None, cu_seqlens=None, convex=False, preprocess=0, workspace=None)
    y, res = add_norm(x, weight, residual=None, scale=1.0, post_weight=None, eps=1e-6)
    y = gate_norm(o, z, weight, activation="silu", eps=1e-6)

The arguments of the functions of the same (or, for glr, the prefill's) name; both
directions run in the library's kernels.  Kept for the backward pass: the operands and
the saved states (glr), the residual stream that add_norm returned, and x where a scale
vector or post_weight is there.  There are first derivatives only: differentiating the
gradients again (create_graph=True, then a second backward pass) raises.
"""

from __future__ import annotations

import torch

from . import layer


def _rows(t):
    """A gradient as the kernels take it: rows of contiguous elements."""
    return t if t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous()


class _Gradients(torch.autograd.Function):
    """The kernels' gradients as results of all that they are formed from: their own
    derivative, which no kernel computes, is an error and not zero."""

    @staticmethod
    def forward(ctx, kernels, *args):
        return kernels(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the recurrence and the block norms have no second derivative: their gradients come "
                           "from kernels and cannot be differentiated again")


def _gradients(kernels, *args):
    """kernels(*args), as part of the backward pass's own graph where one is asked for."""
    return _Gradients.apply(kernels, *args) if torch.is_grad_enabled() else kernels(*args)


class _Glr(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, g, initial_state, cu_seqlens, convex, preprocess, workspace):
        h, final, saved = layer.glr_prefill(x, g, initial_state, cu_seqlens, convex, preprocess,
                                            output_checkpoints=True, workspace=workspace)
        ctx.save_for_backward(x, g, saved, initial_state, cu_seqlens)
        ctx.how = (convex, preprocess, workspace)
        ctx.set_materialize_grads(False)
        return h, final

    @staticmethod
    def backward(ctx, dh, dfinal):
        x, g, saved, s0, cu = ctx.saved_tensors
        convex, preprocess, workspace = ctx.how
        dh = torch.zeros_like(x) if dh is None else _rows(dh)
        dfinal = None if dfinal is None else dfinal.contiguous()
        dx, dg, ds0 = _gradients(layer.glr_backward, dh, x, g, saved, s0, dfinal, cu, convex, preprocess,
                                  workspace)
        return dx, dg, ds0, None, None, None, None


class _AddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, scale, post_weight, eps):
        y, res = layer.add_norm(x, weight, residual, scale, post_weight, eps)
        vector = scale if isinstance(scale, torch.Tensor) else None
        reads_x = vector is not None or post_weight is not None
        ctx.save_for_backward(res, weight, vector, post_weight, x if reads_x else None)
        ctx.how = (scale if vector is None else None, eps, residual is not None, x.dtype)
        ctx.set_materialize_grads(False)
        return y, res

    @staticmethod
    def backward(ctx, dy, dres):
        res, weight, vector, post_weight, x = ctx.saved_tensors
        number, eps, has_residual, dtype = ctx.how
        if dy is None and dres is None:
            return None, None, None, None, None, None
        if dy is None:
            dy = torch.zeros(res.shape, dtype=dtype, device=res.device)
        dres = None if dres is None else _rows(dres)
        dx, dr, dw, ds, dp = _gradients(layer.add_norm_backward, _rows(dy), res, weight, dres, x,
                                        vector if vector is not None else number, post_weight, eps)
        return dx, dw, dr if has_residual else None, ds, dp, None


class _GateNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, o, z, weight, activation, eps):
        ctx.save_for_backward(o, z, weight)
        ctx.how = (activation, eps)
        return layer.gate_norm(o, z, weight, activation, eps)

    @staticmethod
    def backward(ctx, dy):
        o, z, weight = ctx.saved_tensors
        do, dz, dw = _gradients(layer.gate_norm_backward, dy.contiguous(), o, z, weight, *ctx.how)
        return do, dz, dw, None, None


def glr(x, g, initial_state=None, cu_seqlens=None, convex=False, preprocess=0, workspace=None):
    """Differentiable glr_prefill: (h, final state).  Both directions use ``workspace``
    where one is given, and leave their device status in it."""
    return _Glr.apply(x, g, initial_state, cu_seqlens, convex, preprocess, workspace)


def add_norm(x, weight, residual=None, scale=1.0, post_weight=None, eps=1e-6):
    """Differentiable add_norm: (y, residual stream)."""
    return _AddNorm.apply(x, weight, residual, scale, post_weight, eps)


def gate_norm(o, z, weight, activation="silu", eps=1e-6):
    """Differentiable gate_norm."""
    return _GateNorm.apply(o, z, weight, activation, eps)
