"""A normed linear layer whose activations are kept in eight bits for the backward pass, behind torch's autograd.

    y, h = norm_linear(x, gain, weight, residual)
    loss(y, h).backward()

Forward: h = x + residual, the root-mean-square norm of h straight into eight bits, and its product with the weight in eight bits.
Kept for the backward pass are the eight-bit forms that the forward pass made or can make out of the same read -- the norm's output
(the operand of the weight's gradient), h (the checkpoint that the norm's gradient reads) and the transposed weight --, one byte
an element each instead of two or four, and four bytes a row.

Backward: with dy in eight bits along its rows and along its columns out of one read,
    dn = dy W          a product of dy and the transposed weight
    dW = dy^T n        a product of dy^T and the transpose of the kept output, whose values the change of blocks leaves as they are
    dx, dgain          the norm's gradient from the checkpoint of h
Gradients are those of the formulas at the values that eight bits kept; the rounding itself counts as the identity.
"""
from __future__ import annotations

import torch

from . import randes


def _code(t) -> int:
    return randes.BF16 if t.dtype is torch.bfloat16 else randes.F32


class _NormLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, weight, residual, eps):
        needs_weight, needs_input = ctx.needs_input_grad[2], any(ctx.needs_input_grad[i] for i in (0, 1, 3))
        f = randes.rms_norm(x, gain, residual, eps=eps, packed=True, checkpoint=needs_input)
        w, wt = randes.pack8_both(weight) if needs_input else (randes.pack8(weight), None)
        y = randes.packed8_linear(f.y, w, y_dtype=_code(x))
        ctx.save_for_backward(gain, f.y.data if needs_weight else None, f.kept.data if needs_input else None, f.rstd if needs_input else None,
                              wt.data if needs_input else None)
        ctx.shape, ctx.weight_type, ctx.input_type = (x.shape[0], x.shape[1], weight.shape[0]), weight.dtype, _code(x)
        ctx.set_materialize_grads(False)
        return (y, f.h) if residual is not None else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        gain, n8, kept, rstd, wt = ctx.saved_tensors
        n, cols, rows = ctx.shape
        whole = lambda g: None if g is None else g.contiguous()      # (a gradient of a sum arrives expanded)
        dy, dh = whole(dy), whole(dh)
        dx = dgain = dw = None
        if dy is None:
            dx = dh                                              # only the residual stream was used
        else:
            needs_weight, needs_input = n8 is not None, kept is not None
            g, gt = randes.pack8_both(dy) if needs_weight else (randes.pack8(dy), None)
            if needs_weight:
                dw = randes.packed8_linear(gt, randes.pack8_transposed(randes.Packed8Matrix(n, cols, n8))).to(ctx.weight_type)
            if needs_input:
                dn = randes.packed8_linear(g, randes.Packed8Matrix(cols, rows, wt), y_dtype=ctx.input_type)
                dx, dgain = randes.rms_norm_backward(dn, randes.Packed8Matrix(n, cols, kept), rstd, gain, dh=dh)
                dgain = dgain.to(gain.dtype) if ctx.needs_input_grad[1] else None
        need = ctx.needs_input_grad
        return dx if need[0] else None, dgain, dw, dx if need[3] else None, None


def norm_linear(x, gain, weight, residual=None, eps: float = 1e-6):
    """(y, h): h = x + residual (x itself without one), y = (norm of h, times gain) weight^T, differentiable in all of them.

    x, residual: [n, cols] fp32 or bf16 CUDA tensors; gain: [cols] or None; weight: [rows, cols]; y: [n, rows] of x's type.

    A step may be captured into a graph. As with every torch function, warm it up on a side stream and let go of all results of
    eager calls on the same leaves before: a backward pass under capture must not meet an eager graph that still lives."""
    out = _NormLinear.apply(x, gain, weight, residual, float(eps))
    return out if residual is not None else (out, x)
