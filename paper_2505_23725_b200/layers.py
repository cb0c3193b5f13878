"""The operators of the training step as torch autograd functions.

`owner` is a binding.Context or a binding.MuLoCo.  The backward passes are the library's own kernels; nothing
is computed twice and nothing else is kept than what their docstrings in binding.py name.  They are differentiable once,
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
