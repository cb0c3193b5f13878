"""The operators of the training step as torch autograd functions.

`owner` is a binding.Context or a binding.MuLoCo.  The backward passes are the library's own kernels; nothing
else is kept than what their docstrings in binding.py name (so attention's makes the scores again).  They are differentiable once,
in reverse mode: what would need more raises."""
from __future__ import annotations

import torch
from torch.autograd import forward_ad


class _Once(torch.autograd.Function):
    """Hands results on; going back through them raises."""

    @staticmethod
    def forward(ctx, name, n, *tensors):
        ctx.name = name
        return tuple(None if t is None else t.view_as(t) for t in tensors[:n])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name} is differentiable once: the gradients of its gradients are not implemented")


def _dual(t):
    """Whether t carries a forward-mode tangent."""
    return forward_ad.unpack_dual(t).tangent is not None


def _once(name, results, inputs):
    """The results of a backward pass, which are functions of `inputs` without a graph.  Where a graph is being recorded
    (create_graph=True) they get one that raises, so that a loss made from them cannot lose their part silently.  (torch's
    once_differentiable looks at the incoming gradients only: those of y.sum() need none.)  An incoming gradient with a
    forward-mode tangent raises here, as a custom function's dual input does."""
    if torch.is_grad_enabled() or any(t is not None and _dual(t) for t in inputs):
        return _Once.apply(name, len(results), *results, *inputs)
    return results


def _rows(t):
    """t, or a copy of it where the library would refuse its layout: it takes rows of consecutive entries that start on 16 bytes
    and do not overlap, a multiple of 8 entries apart.  Views and the gradients that autograd makes of sums, slices and
    concatenations need not be laid out so."""
    if t.data_ptr() % 16 == 0:
        if t.is_contiguous():
            return t
        if t.dim() == 2 and t.stride(1) == 1 and \
                (t.shape[0] < 2 or (t.stride(0) >= t.shape[1] and t.stride(0) % 8 == 0)):
            return t
    return t.clone(memory_format=torch.contiguous_format)


class _GatedFFN(torch.autograd.Function):
    @staticmethod
    def forward(ctx, owner, activation, save, x, w1, w3, w2):
        y, saved = owner.gated_ffn(x, w1, w3, w2, activation, save=save)
        ctx.owner, ctx.activation = owner, activation
        if save:
            ctx.save_for_backward(x, w1, w3, w2, *saved)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w1, w3, w2, *saved = ctx.saved_tensors
        grads = ctx.owner.gated_ffn_backward(_rows(dy), x, w1, w3, w2, tuple(saved), ctx.activation)
        return (None, None, None, *_once("gated_ffn", grads, (dy, x, w1, w3, w2)))


def gated_ffn(owner, x, w1, w3, w2, activation: str = "silu"):
    """(act(x w1) * (x w3)) w2 over the last dimension of x, differentiable in x and the weights (all bf16)."""
    rows, w1, w3, w2 = _rows(x if x.dim() == 2 else x.reshape(-1, x.shape[-1])), _rows(w1), _rows(w3), _rows(w2)
    # G, U and H are kept only for a backward pass; forward-mode inputs go through the function, which refuses them
    save = torch.is_grad_enabled() and (rows.requires_grad or w1.requires_grad or w3.requires_grad or w2.requires_grad)
    if save or _dual(rows) or _dual(w1) or _dual(w3) or _dual(w2):
        y = _GatedFFN.apply(owner, activation, save, rows, w1, w3, w2)
    else:
        y, _ = owner.gated_ffn(rows, w1, w3, w2, activation, save=False)
    return y if x.dim() == 2 else y.view(*x.shape[:-1], w2.shape[1])


class _QKNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, owner, eps, interleaved, q, k, cos, sin, positions, gain_q, gain_k):
        ctx.owner, ctx.eps, ctx.interleaved = owner, eps, interleaved
        ctx.save_for_backward(q, k, cos, sin, positions, gain_q, gain_k)
        return owner.qk_norm_rope(q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, cos, sin, positions, gain_q, gain_k = ctx.saved_tensors
        # (a tensor that was not given has no gradient)
        dq, dk = (d if d is None or d.stride(2) == 1 else d.contiguous() for d in (dq, dk))
        grads = ctx.owner.qk_norm_rope_backward(dq, dk, q, k, cos, sin, positions, gain_q, gain_k, ctx.eps, ctx.interleaved)
        dq, dk, dgq, dgk = _once("qk_norm_rope", grads, (dq, dk, q, k, cos, sin, gain_q, gain_k))
        return (None, None, None, dq, dk, None, None, None, dgq if gain_q is not None else None,
                dgk if gain_k is not None else None)


def qk_norm_rope(owner, q, k, cos, sin, positions=None, gain_q=None, gain_k=None, eps: float = 1e-6,
                 interleaved: bool = False):
    """Norm and rotation of q [tokens, heads, head_dim] and k (binding.Context.qk_norm_rope), differentiable in q, k
    and the gains.  q or k may be None, and so is its result."""
    return _QKNormRope.apply(owner, eps, interleaved, q, k, cos, sin, positions, gain_q, gain_k)


def _heads(t):
    """t [tokens, heads, head_dim], or a copy of it where the library would refuse its layout (as _rows)."""
    if t.data_ptr() % 16 == 0 and (t.is_contiguous() or (
            t.stride(2) == 1 and all(n < 2 or (s >= t.shape[2] and s % 8 == 0) for n, s in zip(t.shape[:2], t.stride()[:2])))):
        return t
    return t.clone(memory_format=torch.contiguous_format)


class _CausalAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, owner, sequences, scale, q, k, v):
        o, lse = owner.causal_attention(q, k, v, sequences, scale)
        ctx.owner, ctx.sequences, ctx.scale = owner, sequences, scale
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        grads = ctx.owner.causal_attention_backward(_heads(do), q, k, v, o, lse, ctx.sequences, ctx.scale)
        return (None, None, None, *_once("causal_attention", grads, (do, q, k, v)))


def causal_attention(owner, q, k, v, sequences, scale=None):
    """Attention of q [tokens, query heads, head_dim] over k and v [tokens, key heads, head_dim] (bf16), every token over those up to it
    of its own sequence (binding.Sequences of the batch), differentiable in q, k and v."""
    return _CausalAttention.apply(owner, sequences, scale, _heads(q), _heads(k), _heads(v))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, owner, eps, center, x, weight, bias, residual):
        y, h, rstd, mean = owner.layer_norm(x, weight, bias, residual, eps, center)
        ctx.owner, ctx.bias = owner, bias is not None
        ctx.save_for_backward(h, rstd, mean, weight)
        return (y, h) if residual is not None else y

    @staticmethod
    def backward(ctx, dy, dh=None):
        h, rstd, mean, weight = ctx.saved_tensors
        dx, dw, db = ctx.owner.layer_norm_backward(_last(dy), h, rstd, mean, weight, None if dh is None else _last(dh), ctx.bias)
        # The same values for both addends, in a tensor each: whatever hands a gradient on unchanged (a view, a sum) lets a leaf keep
        # it as its own, and in-place work on the one must not reach the other.
        dr = None if not ctx.needs_input_grad[6] else dx.clone() if ctx.needs_input_grad[3] else dx
        dx, dr, dw, db = _once("layer_norm", (dx, dr, dw, db), (dy, dh, h, weight))
        return None, None, None, dx, dw, db, dr


def _last(t):
    """t [tokens, d], or a copy of it where the entries of a row are not consecutive or rows overlap."""
    return t if t.stride(1) == 1 and (t.shape[0] < 2 or t.stride(0) >= t.shape[1]) else t.contiguous()


def layer_norm(owner, x, weight=None, bias=None, residual=None, eps: float = 1e-6, center: bool = True):
    """(h - mean) / sqrt(var + eps) * weight + bias over the last dimension of h = x + residual (center=False: without the mean, the
    root mean square norm), differentiable in x, the residual, weight and bias.  With a residual the result is (y, h): h is
    the stream that goes on."""
    shape = x.shape
    if residual is not None and residual.shape != shape:
        raise ValueError(f"residual must have the shape of x {tuple(shape)} (got {tuple(residual.shape)})")
    x2 = _last(x.reshape(-1, shape[-1]))
    r2 = None if residual is None else _last(residual.reshape(-1, shape[-1]))
    out = _LayerNorm.apply(owner, eps, center, x2, weight, bias, r2)
    return out.view(shape) if residual is None else tuple(t.view(shape) for t in out)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, owner, scale, ids, table):
        ctx.owner, ctx.scale, ctx.rows, ctx.dtype = owner, scale, table.shape[0], table.dtype
        ctx.save_for_backward(ids)
        return owner.embedding(ids, table, scale)

    @staticmethod
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        grad = ctx.owner.embedding_backward(_last(dout), ids, ctx.rows, ctx.scale, ctx.dtype)
        grad, = _once("embedding", (grad,), (dout,))
        return None, None, None, grad


def embedding(owner, ids, table, scale: float = 1.0):
    """scale * table[ids] for int64 ids of any shape, differentiable in the table (the gradient, of the table's type, has every row)."""
    out = _Embedding.apply(owner, scale, ids.reshape(-1).contiguous(), _last(table))
    return out.view(*ids.shape, table.shape[1])
