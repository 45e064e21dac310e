"""The residual feed-forward block between two masked boundaries, as autograd
ops (paper Sec. 3.1; Alg. 1: a stage runs its layers on the unpacked
activation, and its weight gradients go to the corrector).

    out = x + W2 act(W1 norm(x) + b1) + b2

mlp_block is one autograd node.  What it keeps for the backward pass is the
block's input and the hidden pre-activation, each as an 8-bit checkpoint that
the norm and the product write in their own pass (1.03 bytes a value), or
whole (checkpoint=False).  The norm's output and the hidden activation are
computed again from them.  layer_norm and linear are its parts as nodes of
their own, for blocks of another form.

The ops are differentiable once: the gradient of a gradient raises an error.
Gradients of W1 and W2 come out in the weights' dtype, as sc_correct takes
them.  Every operation is a library call; this module only wires them into
autograd.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import (Q8, lin_backward_act, lin_backward_input, lin_backward_weight, lin_forward, ln_backward, ln_forward,
               ln_recompute)


def _flat(t: torch.Tensor) -> torch.Tensor:
    """[rows, H] with unit column stride."""
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 and (t.shape[0] < 2 or t.stride(0) >= t.shape[1]) else t.contiguous()


def _save(src):
    return tuple(src) if isinstance(src, Q8) else (src, None)


def _load(a, b):
    return a if b is None else Q8(a, b)


def _as(t, like):
    return None if t is None or like is None else t.to(like.dtype)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, eps: float, checkpoint: bool):
        x2 = _flat(x)
        y, mean, rstd, q = ln_forward(x2, gamma, beta, eps, checkpoint=checkpoint)
        ctx.save_for_backward(mean, rstd, gamma, beta, *_save(q if checkpoint else x2))
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        mean, rstd, gamma, beta, a, b = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dgamma, dbeta = ln_backward(_flat(g), _load(a, b), mean, rstd, gamma, weights=need[1] or need[2])
        return dx.view(g.shape), _as(dgamma, gamma), _as(dbeta, beta), None, None


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, bias, residual, act: str, checkpoint: bool):
        x2 = _flat(x)
        r2 = _flat(residual) if residual is not None else None
        keep = None if act == "none" else ("q8" if checkpoint else "z")
        y, z = lin_forward(x2, W, bias, act, r2, keep)
        ctx.act = act
        ctx.save_for_backward(x2, W, bias, *_save(z))
        ctx.residual = None if residual is None else residual.shape
        return y.view(*x.shape[:-1], W.shape[0])

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        x2, W, bias, a, b = ctx.saved_tensors
        need = ctx.needs_input_grad
        dz = g2 = _flat(g)
        if ctx.act != "none" and any(need[:3]):
            dz = lin_backward_act(g2, _load(a, b), ctx.act)
        dx = dW = db = None
        if need[0]:
            dx = lin_backward_input(dz, W).view(*g.shape[:-1], W.shape[1])
        if need[1] or need[2]:
            dW, db = lin_backward_weight(dz, x2, bias=need[2])
        return dx, dW, _as(db, bias), g.reshape(ctx.residual) if need[3] else None, None, None


class _MlpBlock(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, W1, b1, W2, b2, act: str, eps: float, checkpoint: bool):
        x2 = _flat(x)
        y, mean, rstd, q = ln_forward(x2, gamma, beta, eps, checkpoint=checkpoint)
        a, z = lin_forward(y, W1, b1, act, keep="q8" if checkpoint else "z")
        out, _ = lin_forward(a, W2, b2, residual=x2)
        ctx.act = act
        ctx.save_for_backward(mean, rstd, gamma, beta, W1, b1, W2, b2, *_save(q if checkpoint else x2), *_save(z))
        return out.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        mean, rstd, gamma, beta, W1, b1, W2, b2, *kept = ctx.saved_tensors
        x, z = _load(*kept[:2]), _load(*kept[2:])
        g2 = _flat(g)
        need = ctx.needs_input_grad
        dx = dgamma = dbeta = dW1 = db1 = dW2 = db2 = None
        if need[5] or need[6]:
            dW2, db2 = lin_backward_weight(g2, z, act=ctx.act, bias=need[6])
        if any(need[:5]):
            dz = lin_backward_input(g2, W2, act=ctx.act, z=z)
            if need[3] or need[4]:
                y = ln_recompute(x, mean, rstd, gamma, beta, dtype=g2.dtype)
                dW1, db1 = lin_backward_weight(dz, y, bias=need[4])
                del y
            if any(need[:3]):
                dy = lin_backward_input(dz, W1)
                dx, dgamma, dbeta = ln_backward(dy, x, mean, rstd, gamma, add=g2, weights=need[1] or need[2])
                dx = dx.view(g.shape)
        return (dx, _as(dgamma, gamma), _as(dbeta, beta), dW1, _as(db1, b1), dW2, _as(db2, b2), None, None, None)


def layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, checkpoint: bool = False):
    """Layer norm over the last dimension; checkpoint keeps x in 8 bits."""
    return _LayerNorm.apply(x, gamma, beta, float(eps), bool(checkpoint))


def linear(x, W, bias=None, act: str = "none", residual=None, checkpoint: bool = False):
    """act(x W^T + bias) + residual; checkpoint keeps the pre-activation in 8
    bits (the input is kept whole: it is another op's output)."""
    return _Linear.apply(x, W, bias, residual, act, bool(checkpoint))


def mlp_block(x, gamma, beta, W1, b1, W2, b2, act: str = "gelu", eps: float = 1e-5, checkpoint: bool = True):
    """x + W2 act(W1 norm(x) + b1) + b2 for x [..., H], W1 [F, H], W2 [H, F]."""
    return _MlpBlock.apply(x, gamma, beta, W1, b1, W2, b2, act, float(eps), bool(checkpoint))
