"""Attention, layer norm and embedding without a GPU: struct layouts, refusals without a context, the definitions that the GPU tests
compare with against differences, and what the autograd forms pass on, refuse and hand out over a stand-in owner."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2505_23725_b200 import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2505_23725_b200 import binding as B
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "muloco.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu %zu %d\\n", sizeof(muloco_attention), sizeof(muloco_norm),'
                   ' sizeof(muloco_embedding), offsetof(muloco_attention, q), offsetof(muloco_attention, v_head_stride),'
                   ' offsetof(muloco_norm, eps), offsetof(muloco_norm, bias), offsetof(muloco_embedding, ids),'
                   ' MULOCO_NORM_PARTS); return 0;}\n')
    exe = tmp_path / "t"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).decode().split()]
    assert out == [C.sizeof(B.Attention), C.sizeof(B.Norm), C.sizeof(B.Embedding), B.Attention.q.offset,
                   B.Attention.v_head_stride.offset, B.Norm.eps.offset, B.Norm.bias.offset, B.Embedding.ids.offset, B.NORM_PARTS]
    a = B.Attention.from_buffer_copy(B._ATTENTION_PACK(4, 2, 64, 0.5, *range(10, 19)))
    assert (a.heads_q, a.heads_k, a.head_dim, a.scale, a.q, a.v, a.q_token_stride, a.v_head_stride) == (4, 2, 64, 0.5, 10, 12, 13, 18)
    a = B.Norm.from_buffer_copy(B._NORM_PACK(1, 2, 3, 4, 1, 0, 0.25, 0, *range(10, 14)))
    assert (a.tokens, a.d, a.ldx, a.ldr, a.dtype, a.center, a.eps, a.x, a.residual, a.weight, a.bias) == \
        (1, 2, 3, 4, 1, 0, 0.25, 10, 11, 12, 13)
    a = B.Embedding.from_buffer_copy(B._EMBEDDING_PACK(1, 2, 3, 4, 1, 0.5, 10))
    assert (a.tokens, a.rows, a.d, a.ld, a.dtype, a.scale, a.ids) == (1, 2, 3, 4, 1, 0.5, 10)


def test_a_null_context_is_an_argument_error():
    from paper_2505_23725_b200 import binding as B
    lib = B.load_library()
    assert lib.muloco_sequences_bytes(None, None, 0, 0, None) == B.EINVAL
    assert lib.muloco_sequences_create(None, None, 0, 0, None, 0, None) == B.EINVAL
    lib.muloco_sequences_destroy(None)
    assert lib.muloco_causal_attention(None, b"", None, None, None) == B.EINVAL
    assert lib.muloco_causal_attention_backward(None, b"", None, None, 0, 0, *[None] * 6) == B.EINVAL
    assert lib.muloco_layer_norm(None, b"", None, None, None, None) == B.EINVAL
    assert lib.muloco_layer_norm_backward(None, b"", None, 0, *[None] * 6) == B.EINVAL
    assert lib.muloco_embedding_lookup(None, b"", None, None) == B.EINVAL
    assert lib.muloco_embedding_scratch(None, 1, 1, None) == B.EINVAL
    assert lib.muloco_embedding_backward(None, b"", None, 0, None, None) == B.EINVAL


def _differences(f, x, h=1e-6):
    d = torch.zeros_like(x)
    for i in range(x.numel()):
        y, z = x.clone(), x.clone()
        y.view(-1)[i] += h
        z.view(-1)[i] -= h
        d.view(-1)[i] = (f(y) - f(z)) / (2 * h)
    return d


@pytest.mark.parametrize("lengths,hq,hk", [([1], 1, 1), ([3, 0, 4], 4, 2), ([5], 3, 1)])
def test_definition_of_attention_against_differences(lengths, hq, hk):
    from test_gpu_attention import reference
    torch.manual_seed(0)
    T, D = sum(lengths) + 1, 6
    q, k, v, do = (torch.randn(T, h, D, dtype=torch.float64) for h in (hq, hk, hk, hq))
    r, _ = reference(q, k, v, do, lengths, 0.4)
    for name, t, f in (("dq", q, lambda x: reference(x, k, v, do, lengths, 0.4)), ("dk", k, lambda x: reference(q, x, v, do, lengths, 0.4)),
                       ("dv", v, lambda x: reference(q, k, x, do, lengths, 0.4))):
        assert torch.allclose(r[name], _differences(lambda x: (f(x)[0]["o"] * do).sum(), t), atol=1e-7)
    # the plain loop over pairs
    o = torch.zeros_like(q)
    at = 0
    for n in lengths:
        for i in range(n):
            for h in range(hq):
                w = torch.stack([(q[at + i, h] @ k[at + j, h * hk // hq] * 0.4).exp() for j in range(i + 1)])
                o[at + i, h] = sum(w[j] * v[at + j, h * hk // hq] for j in range(i + 1)) / w.sum()
        at += n
    assert torch.allclose(o, r["o"], atol=1e-12)


# ------------------------------------------------------------------------------------------------
# autograd forms over a stand-in owner
# ------------------------------------------------------------------------------------------------
class Owner:
    """float64 in place of the library's types; a layout that it would answer with an error raises."""

    def _heads(self, t):
        for n, s in zip(t.shape[:2], t.stride()[:2]):
            if n > 1 and (s < t.shape[2] or s % 8):
                raise RuntimeError(f"ESHAPE: strides {t.stride()}")
        assert t.stride(2) == 1 and t.data_ptr() % 16 == 0

    def causal_attention(self, q, k, v, sequences, scale=None):
        from test_gpu_attention import reference
        for t in (q, k, v):
            self._heads(t)
        r, _ = reference(q.detach(), k.detach(), v.detach(), torch.zeros_like(q), sequences, scale)
        return r["o"], r["lse"]

    def causal_attention_backward(self, do, q, k, v, o, lse, sequences, scale=None):
        from test_gpu_attention import reference
        for t in (do, q, k, v):
            self._heads(t)
        assert o.is_contiguous()
        r, _ = reference(q.detach(), k.detach(), v.detach(), do.detach(), sequences, scale)
        return r["dq"], r["dk"], r["dv"]

    def layer_norm(self, x, weight=None, bias=None, residual=None, eps=1e-6, center=True):
        with torch.no_grad():
            for t in (x, residual):
                assert t is None or t.stride(1) == 1
            h = x if residual is None else x + residual
            mean = h.mean(1) if center else None
            z = h - mean[:, None] if center else h
            rstd = (z.square().mean(1) + eps).rsqrt()
            y = z * rstd[:, None] * (1 if weight is None else weight) + (0 if bias is None else bias)
            return y, h, rstd, mean

    def layer_norm_backward(self, dy, h, rstd, mean=None, weight=None, dh=None, bias=False):
        with torch.no_grad():
            for t in (dy, dh):
                assert t is None or t.stride(1) == 1
            n = (h - (0 if mean is None else mean[:, None])) * rstd[:, None]
            e = dy * (1 if weight is None else weight)
            dx = e - n * (e * n).mean(1, keepdim=True) - (0 if mean is None else e.mean(1, keepdim=True))
            dx = dx * rstd[:, None] + (0 if dh is None else dh)
            return dx, (dy * n).sum(0) if weight is not None else None, dy.sum(0) if bias else None

    def embedding(self, ids, table, scale=1.0):
        assert ids.is_contiguous() and table.stride(1) == 1
        return table.detach()[ids] * scale

    def embedding_backward(self, dout, ids, rows, scale=1.0, dtype=None):
        assert dout.stride(1) == 1 and dout.dtype == dtype
        return torch.zeros(rows, dout.shape[1], dtype=dtype).index_add_(0, ids, dout.detach()) * scale


def rand(*shape, grad=True):
    return torch.randn(*shape, dtype=torch.float64).requires_grad_(grad)


@pytest.mark.parametrize("layout", ["dense", "fused", "head dimension first"])
def test_attention_under_autograd(layout):
    torch.manual_seed(1)
    lengths, T, D = [3, 2], 6, 8
    if layout == "fused":
        base = [rand(T, 4, D)]
        make = lambda b: (b[0][:, :2], b[0][:, 2:3], b[0][:, 3:])                 # noqa: E731
    elif layout == "head dimension first":
        base = [rand(D, T, 2), rand(D, T, 1), rand(D, T, 1)]
        make = lambda b: tuple(t.permute(1, 2, 0) for t in b)                     # noqa: E731
    else:
        base = [rand(T, 2, D), rand(T, 1, D), rand(T, 1, D)]
        make = lambda b: tuple(b)                                                 # noqa: E731
    weight = torch.randn(D, 2, T, dtype=torch.float64).permute(2, 1, 0)           # an incoming gradient of another layout

    def loss(b):
        return (layers.causal_attention(Owner(), *make(b), lengths, 0.5) * weight).sum()

    grads = torch.autograd.grad(loss(base), base)
    for i, (g, b) in enumerate(zip(grads, base)):
        def f(x):
            return loss([x if j == i else t.detach() for j, t in enumerate(base)]).detach()
        assert torch.allclose(g, _differences(f, b.detach()), atol=1e-7)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("use", ["y", "h", "both", "without residual"])
def test_norm_under_autograd(center, use):
    torch.manual_seed(2)
    x, r, w, b = rand(2, 3, 5), rand(2, 3, 5), rand(5), rand(5)
    cy, ch = torch.randn(2, 3, 5, dtype=torch.float64), torch.randn(5, 3, 2, dtype=torch.float64).permute(2, 1, 0)

    def loss(x, w, b, r):
        if use == "without residual":
            return (layers.layer_norm(Owner(), x, w, b, eps=1e-3, center=center) * cy).sum() + 0.0 * r.sum()
        y, h = layers.layer_norm(Owner(), x, w, b, residual=r, eps=1e-3, center=center)
        assert y.shape == h.shape == x.shape
        return (y * cy).sum() * (use != "h") + (h * ch).sum() * (use != "y")

    args = [x, w, b, r]
    grads = torch.autograd.grad(loss(*args), args)
    for i, g in enumerate(grads):
        def f(t):
            return loss(*[t if j == i else a.detach() for j, a in enumerate(args)]).detach()
        assert torch.allclose(g, _differences(f, args[i].detach()), atol=1e-7)


def test_gradients_of_one_sum_do_not_share_memory():
    x, r = rand(4, 6), rand(4, 6)
    y, h = layers.layer_norm(Owner(), x, residual=r)
    (y.sum() + (h * h).sum()).backward()
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()


def test_embedding_under_autograd():
    torch.manual_seed(3)
    table = rand(7, 8)
    ids = torch.tensor([[1, 5, 1], [0, 1, 6]])
    out = layers.embedding(Owner(), ids.T, table, 0.5)
    assert out.shape == (3, 2, 8) and torch.equal(out, table[ids.T] * 0.5)
    c = torch.randn(8, 2, 3, dtype=torch.float64).permute(2, 1, 0)
    g, = torch.autograd.grad((out * c).sum(), table)
    want, = torch.autograd.grad((table[ids.T] * 0.5 * c).sum(), table)
    assert torch.allclose(g, want)


def test_gradients_of_gradients_raise():
    table, x = rand(7, 8), rand(4, 8)
    q, k, v = rand(3, 2, 8), rand(3, 1, 8), rand(3, 1, 8)
    for out, leaf in ((layers.embedding(Owner(), torch.tensor([1, 2]), table), table), (layers.layer_norm(Owner(), x, rand(8)), x),
                      (layers.causal_attention(Owner(), q, k, v, [3], 1.0), q)):
        g, = torch.autograd.grad(out.square().sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiable once"):
            g.square().sum().backward()
