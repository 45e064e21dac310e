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

glu_block is the block of models with root-mean-square norms, a gated product
and, where they have them, a norm after the block, gains of its gate, dropout
and a scaled residual:

    h = act(Wg norm(x) + bg) (Wu norm(x) + bu)
    out = scale x + D(gate norm(W2 h + b2))

rms_norm, glu, dropout and join are its parts; join also takes the norm before
the next block into its pass.  A dropout's mask comes from its key in both
passes, and is kept nowhere.

The ops are differentiable once: the gradient of a gradient raises an error.
Gradients of W1 and W2 come out in the weights' dtype, as sc_correct takes
them.  The gated product's bias gradient is summed before its terms are rounded;
that of a linear layer from the gradient that reaches it, in its tensor's dtype.
Every operation is a library call; this module only wires them into autograd.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import (Q8, drop_apply, glu_backward_act, glu_backward_act_bias, glu_backward_input, glu_forward, join_backward, join_forward,
               lin_backward_act, lin_backward_input, lin_backward_weight, lin_forward, ln_backward, ln_forward, ln_recompute,
               rms_backward, rms_forward, rms_recompute)


def _flat(t: torch.Tensor) -> torch.Tensor:
    """[rows, H] with unit column stride."""
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 and (t.shape[0] < 2 or t.stride(0) >= t.shape[1]) else t.contiguous()


def _save(src):
    return tuple(src) if isinstance(src, Q8) else (src, None)


def _load(a, b):
    return a if b is None else Q8(a, b)


def _save_pair(z):
    """Kept pre-activations of the gated product: one tensor, or two checkpoints."""
    return (z, None, None, None) if isinstance(z, torch.Tensor) else (*z[0], *z[1])


def _load_pair(t):
    return t[0] if t[1] is None else (Q8(t[0], t[1]), Q8(t[2], t[3]))


def _keep(checkpoint, *ts):
    """How an op keeps what its backward pass reads: in 8 bits (True), whole
    (False), or not at all (None), where no gradient is wanted."""
    return bool(checkpoint) if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in ts) else None


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


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, eps: float, keep):
        x2 = _flat(x)
        y, rstd, q = rms_forward(x2, gamma, eps, checkpoint=bool(keep))
        if keep is not None:
            ctx.save_for_backward(rstd, gamma, *_save(q if keep else x2))
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        rstd, gamma, a, b = ctx.saved_tensors
        dx, dgamma = rms_backward(_flat(g), _load(a, b), rstd, gamma, weights=ctx.needs_input_grad[1])
        return dx.view(g.shape), _as(dgamma, gamma), None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, drop):
        ctx.drop = drop
        ctx.residual = None if residual is None else residual.shape
        return drop_apply(_flat(x), drop, None if residual is None else _flat(residual)).view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        dx = drop_apply(_flat(g), ctx.drop).view(g.shape) if ctx.needs_input_grad[0] else None
        return dx, g.reshape(ctx.residual) if ctx.needs_input_grad[1] else None, None


class _Join(torch.autograd.Function):
    @staticmethod
    def forward(ctx, r, b, post, gate, pre, scale: float, drop, eps: float, keep):
        r2, b2 = _flat(r), _flat(b)
        branch = post is not None or gate is not None
        # of what the backward pass reads
        parts = bool(keep) and {(1, 1): True, (1, 0): "out", (0, 1): "b", (0, 0): False}[pre is not None, branch]
        j = join_forward(r2, b2, post, gate, pre, scale, drop, eps, parts)
        if keep is not None:
            src_out = None if pre is None else j.q_out if keep else j.out
            src_b = None if not branch else j.q_b if keep else b2
            ctx.save_for_backward(post, gate, pre, j.rstd_post, j.rstd_pre, *_save(src_out), *_save(src_b))
        ctx.scale, ctx.drop, ctx.shapes = scale, drop, (r.shape, b.shape)
        ctx.set_materialize_grads(False)
        out = j.out.view(r.shape)
        return out if pre is None else (out, j.y.view(r.shape))

    @staticmethod
    @once_differentiable
    def backward(ctx, gout, gy=None):
        post, gate, pre, rstd_post, rstd_pre, *kept = ctx.saved_tensors
        need = ctx.needs_input_grad
        if gout is None and gy is None:
            return (None,) * 9
        d = join_backward(None if gout is None else _flat(gout), None if gy is None else _flat(gy), _load(*kept[:2]),
                          _load(*kept[2:]), rstd_post, rstd_pre, post, gate, pre, ctx.scale, ctx.drop,
                          weights=_wanted(need[2:5]), want_dr=need[0])
        return (d.dr.view(ctx.shapes[0]) if need[0] else None, d.db.view(ctx.shapes[1]), _as(d.dpost, post), _as(d.dgate, gate),
                _as(d.dpre, pre), None, None, None, None)


def _wanted(need):
    """The gains whose gradients are wanted, as join_backward names them."""
    return tuple(name for name, k in zip(("post", "gate", "pre"), need) if k)


_GLU_KEEP = {True: "q8", False: "z", None: None}


class _Glu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, bias, act: str, keep):
        x2 = _flat(x)
        h, z = glu_forward(x2, W, bias, act, _GLU_KEEP[keep])
        ctx.act = act
        if keep is not None:
            ctx.save_for_backward(x2, W, bias, *_save_pair(z))
        return h.view(*x.shape[:-1], h.shape[1])

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        x2, W, bias, *kept = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dW = db = None
        if any(need[:3]):
            if need[2]:
                dz, _, db = glu_backward_act_bias(_flat(g), _load_pair(kept), ctx.act)
            else:
                dz, _ = glu_backward_act(_flat(g), _load_pair(kept), ctx.act)
            if need[0]:
                dx = lin_backward_input(dz, W).view(*g.shape[:-1], W.shape[1])
            if need[1]:
                dW, _ = lin_backward_weight(dz, x2, bias=False)
        return dx, dW, _as(db, bias), None, None


class _GluBlock(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, W, bias, W2, bias2, post, gate, scale: float, drop, act: str, eps: float, keep):
        x2 = _flat(x)
        y, rstd, q = rms_forward(x2, gamma, eps, checkpoint=bool(keep))
        h, z = glu_forward(y, W, bias, act, _GLU_KEEP[keep])
        ctx.plain = post is None and gate is None and drop is None and scale == 1.0
        rstd_post = b = None
        if ctx.plain:
            out, _ = lin_forward(h, W2, bias2, residual=x2)
        else:
            b, _ = lin_forward(h, W2, bias2)
            branch = post is not None or gate is not None
            j = join_forward(x2, b, post, gate, None, scale, drop, eps, "b" if keep and branch else False)
            out, rstd_post = j.out, j.rstd_post
            b = None if not branch else j.q_b if keep else b
        ctx.scale, ctx.drop, ctx.act = scale, drop, act
        if keep is not None:
            ctx.save_for_backward(rstd, gamma, W, bias, W2, bias2, post, gate, rstd_post, *_save(q if keep else x2), *_save(b),
                                  *_save_pair(z))
        return out.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        rstd, gamma, W, bias, W2, bias2, post, gate, rstd_post, *kept = ctx.saved_tensors
        x, b, z = _load(*kept[:2]), _load(*kept[2:4]), _load_pair(kept[4:])
        need = ctx.needs_input_grad
        dx = dgamma = dW = dbias = dW2 = dbias2 = dpost = dgate = None
        dr = db = _flat(g)
        if not ctx.plain:
            # where the stream is not scaled its gradient is g itself
            scaled = need[0] and ctx.scale != 1.0
            d = join_backward(db, None, None, b, rstd_post, None, post, gate, None, ctx.scale, ctx.drop, weights=_wanted(need[6:8]),
                              want_dr=scaled)
            db, dpost, dgate = d.db, d.dpost, d.dgate
            if scaled:
                dr = d.dr
        dz = h = None
        if any(need[:6]):
            dz, h, dbias = glu_backward_input(db, W2, z, ctx.act, hidden=need[4] or need[5], bias=need[3])
        if need[4] or need[5]:
            dW2, dbias2 = lin_backward_weight(db, h, bias=need[5])
        del h
        if need[2]:
            y = rms_recompute(x, rstd, gamma, dtype=db.dtype)
            dW, _ = lin_backward_weight(dz, y, bias=False)
            del y
        if need[0] or need[1]:
            dx, dgamma = rms_backward(lin_backward_input(dz, W), x, rstd, gamma, add=dr if need[0] else None, weights=need[1])
            dx = dx.view(g.shape)
        return (dx, _as(dgamma, gamma), dW, _as(dbias, bias), dW2, _as(dbias2, bias2), _as(dpost, post), _as(dgate, gate), None,
                None, None, None, None)


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


def rms_norm(x, gamma=None, eps: float = 1e-5, checkpoint: bool = False):
    """Root-mean-square norm over the last dimension; checkpoint keeps x in 8 bits."""
    return _RmsNorm.apply(x, gamma, float(eps), _keep(checkpoint, x, gamma))


def dropout(x, drop, residual=None):
    """D(x) + residual for x [..., H]; drop: a Drop whose key has x's rows."""
    return _Dropout.apply(x, residual, drop)


def join(r, b, post=None, gate=None, pre=None, scale: float = 1.0, drop=None, eps: float = 1e-5, checkpoint: bool = False):
    """Between two blocks: out = scale r + D(gate norm(b)), with post the gains
    of the norm (None: b as it is); with pre, (out, norm(out)), the input of the
    next block, from the same pass.  checkpoint keeps out and b in 8 bits."""
    return _Join.apply(r, b, post, gate, pre, float(scale), drop, float(eps), _keep(checkpoint, r, b, post, gate, pre))


def glu(x, W, bias=None, act: str = "silu", checkpoint: bool = False):
    """act(x Wg^T + bg) (x Wu^T + bu), W [2 F, H] with Wg's rows first;
    checkpoint keeps the pre-activations in 8 bits."""
    return _Glu.apply(x, W, bias, act, _keep(checkpoint, x, W, bias))


def glu_block(x, gamma, W, bias, W2, bias2, post=None, gate=None, scale: float = 1.0, drop=None, act: str = "silu",
              eps: float = 1e-5, checkpoint: bool = True):
    """scale x + D(gate norm(W2 h + bias2)), h = glu(norm(x)), for x [..., H],
    W [2 F, H], W2 [H, F].  gamma, post: the gains of the norms before and after
    (post None: no norm after); biases, gate and drop may be None."""
    return _GluBlock.apply(x, gamma, W, bias, W2, bias2, post, gate, float(scale), drop, act, float(eps),
                           _keep(checkpoint, x, gamma, W, bias, W2, bias2, post, gate))
