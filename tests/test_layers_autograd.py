"""layers.py without a GPU: what the autograd forms pass on, refuse and hand out, over a stand-in owner that computes the
operators in plain torch and takes only the layouts that the library takes."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2505_23725_b200 import layers


def _silu_parts(g):
    s = torch.sigmoid(g)
    return g * s, s * (1 + g * (1 - s))


class Owner:
    """float64 in place of bf16; a layout that the library would answer with an error raises."""

    def _rows(self, t):
        t_ok = t.stride(1) == 1 and t.data_ptr() % 16 == 0 and t.shape[1] % 8 == 0
        if not t_ok or (t.shape[0] > 1 and (t.stride(0) < t.shape[1] or t.stride(0) % 8 != 0)):
            raise RuntimeError(f"ESHAPE: strides {t.stride()}")

    def gated_ffn(self, x, w1, w3, w2, activation="silu", save=True):
        for t in (x, w1, w3, w2):
            self._rows(t)
        with torch.no_grad():
            g, u = x.detach() @ w1.detach(), x.detach() @ w3.detach()
            h = _silu_parts(g)[0] * u
            return h @ w2.detach(), ((g, u, h) if save else None)

    def gated_ffn_backward(self, dy, x, w1, w3, w2, saved, activation="silu"):
        for t in (dy, x, w1, w3, w2):
            self._rows(t)
        with torch.no_grad():
            dy, x, w1, w3, w2 = (t.detach() for t in (dy, x, w1, w3, w2))
            g, u, h = saved
            value, slope = _silu_parts(g)
            dh = dy @ w2.T
            dg, du = dh * u * slope, dh * value
            return dg @ w1.T + du @ w3.T, x.T @ dg, x.T @ du, h.T @ dy

    # the "norm" of the stand-in: x -> gain * x
    def qk_norm_rope(self, q, k, cos, sin, positions=None, gain_q=None, gain_k=None, eps=1e-6, interleaved=False):
        with torch.no_grad():
            return tuple(None if x is None else x * (1 if g is None else g) for x, g in ((q, gain_q), (k, gain_k)))

    def qk_norm_rope_backward(self, dq, dk, q, k, cos, sin, positions=None, gain_q=None, gain_k=None, eps=1e-6, interleaved=False):
        out, gains = [], []
        with torch.no_grad():
            for d, x, g in ((dq, q, gain_q), (dk, k, gain_k)):
                assert (d is None) == (x is None)
                assert d is None or d.stride(2) == 1
                out.append(None if x is None else d * (1 if g is None else g))
                gains.append(None if x is None else (d * x).sum((0, 1)))
        return (*out, *gains)


def _tensors(T=3, d=8, F=16, grad=True):
    torch.manual_seed(0)
    return [(torch.randn(*s, dtype=torch.float64) / 2).requires_grad_(grad) for s in ((T, d), (d, F), (d, F), (F, d))]


def _plain(x, w1, w3, w2):
    return (_silu_parts(x @ w1)[0] * (x @ w3)) @ w2


def _qk(T=3, h=2, D=4, grad=True):
    torch.manual_seed(1)
    q, k = (torch.randn(T, h, D, dtype=torch.float64, requires_grad=grad) for _ in range(2))
    gq, gk = (torch.randn(D, dtype=torch.float64, requires_grad=grad) for _ in range(2))
    return q, k, torch.ones(T, D // 2), torch.zeros(T, D // 2), None, gq, gk


# -- second derivatives -------------------------------------------------------------------------
@pytest.mark.parametrize("loss", [lambda y: y.sum(), lambda y: y.square().sum()], ids=["linear", "square"])
def test_second_derivatives_are_refused_not_dropped(loss):
    """The backward kernels have no graph of their own.  A gradient taken with create_graph=True can be used as a number,
    but differentiating it says so instead of returning a gradient without that term."""
    args = _tensors()
    y = layers.gated_ffn(Owner(), *args)
    grads = torch.autograd.grad(loss(y), args, create_graph=True)
    want = torch.autograd.grad(loss(_plain(*args)), args)
    assert all(torch.allclose(a, b) for a, b in zip(grads, want))
    penalty = sum(g.square().sum() for g in grads)
    assert penalty.requires_grad
    with pytest.raises(RuntimeError, match="once"):
        (args[0].square().sum() + penalty).backward()

    q, k, cos, sin, _, gq, gk = _qk()
    a, b = layers.qk_norm_rope(Owner(), q, k, cos, sin, None, gq, gk)
    grads = torch.autograd.grad(loss(a) + loss(b), (q, k, gq, gk), create_graph=True)
    for g in grads:
        assert g.requires_grad
        with pytest.raises(RuntimeError, match="once"):
            (q.sum() + g.sum()).backward(retain_graph=True)


def test_first_derivatives_with_create_graph_reach_the_rest_of_the_graph():
    """create_graph=True with the block in the graph: derivatives that do not pass through its gradient still work."""
    x, *ws = _tensors()
    z = torch.randn(3, 8, dtype=torch.float64, requires_grad=True)
    loss = layers.gated_ffn(Owner(), x, *ws).sum() + (z ** 3).sum()
    gx, gz = torch.autograd.grad(loss, (x, z), create_graph=True)
    gz.sum().backward()
    assert torch.allclose(z.grad, 6 * z) and torch.allclose(gx, torch.autograd.grad(_plain(x, *ws).sum(), x)[0])


def test_first_derivatives():
    args = _tensors()
    layers.gated_ffn(Owner(), *args).square().sum().backward()
    want = torch.autograd.grad(_plain(*args).square().sum(), args)
    assert all(torch.allclose(t.grad, g) and not t.grad.requires_grad for t, g in zip(args, want))


# -- forward mode -------------------------------------------------------------------------------
@pytest.mark.parametrize("grad", [False, True], ids=["no_grad", "grad"])
@pytest.mark.parametrize("which", range(4))
def test_forward_mode_is_refused_not_dropped(grad, which):
    args = _tensors(grad=False)
    qk = _qk(grad=False)
    at = (0, 1, 5, 6)[which]
    with torch.set_grad_enabled(grad), forward_ad.dual_level():
        duals = list(args)
        duals[which] = forward_ad.make_dual(args[which], torch.ones_like(args[which]))
        with pytest.raises(NotImplementedError, match="forward mode"):
            layers.gated_ffn(Owner(), *duals)
        duals = list(qk)
        duals[at] = forward_ad.make_dual(qk[at], torch.ones_like(qk[at]))
        with pytest.raises(NotImplementedError, match="forward mode"):
            layers.qk_norm_rope(Owner(), *duals)


def test_tangents_of_incoming_gradients_are_refused():
    args = _tensors()
    y = layers.gated_ffn(Owner(), *args)
    q, k, *rest = _qk()
    a, _ = layers.qk_norm_rope(Owner(), q, k, *rest)
    with forward_ad.dual_level():
        for out, at in ((y, args[0]), (a, q)):
            dy = forward_ad.make_dual(torch.ones_like(out), torch.ones_like(out))
            with pytest.raises(NotImplementedError, match="forward mode"):
                torch.autograd.grad(out, at, dy, retain_graph=True)


def test_nothing_is_kept_where_no_gradient_is_wanted():
    class Watched(Owner):
        saves = []

        def gated_ffn(self, x, w1, w3, w2, activation="silu", save=True):
            self.saves.append(save)
            return super().gated_ffn(x, w1, w3, w2, activation, save)

    args = _tensors()
    o = Watched()
    layers.gated_ffn(o, *args)
    with torch.no_grad():
        y = layers.gated_ffn(o, *args)
    z = layers.gated_ffn(o, *(t.detach() for t in args))
    with torch.inference_mode():
        layers.gated_ffn(o, *(t.detach() for t in args))
    assert o.saves == [True, False, False, False] and not y.requires_grad and not z.requires_grad
    assert torch.allclose(y, _plain(*args)) and torch.equal(y, z)


# -- layouts ------------------------------------------------------------------------------------
LOSSES = {
    "sum over tokens": lambda y: (y.sum(0) * torch.arange(8.0, dtype=torch.float64)).sum(),     # strides (0, 1)
    "sum": lambda y: y.sum(),                                                                    # strides (0, 0)
    "cat of an odd width": lambda y: (torch.cat([y, y.detach()[:, :3]], 1) ** 2).sum(),          # row stride 11
    "cat behind an odd width": lambda y: (torch.cat([y.detach()[:, :3], y], 1) ** 2).sum(),      # ... and off 16 bytes
    "transposed": lambda y: (y.t().contiguous() ** 2).sum(),
}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("T", [1, 3])
def test_gradients_of_any_layout(loss, T):
    args = _tensors(T)
    got = torch.autograd.grad(LOSSES[loss](layers.gated_ffn(Owner(), *args)), args)
    want = torch.autograd.grad(LOSSES[loss](_plain(*args)), args)
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


def _views(t):
    """t as parts of wider matrices, transposed, at an odd address, expanded from one row."""
    n, m = t.shape
    yield torch.cat([t, t[:, :3]], 1)[:, :m]
    yield torch.cat([t[:, :1], t, t[:, :7]], 1)[:, 1:m + 1]
    yield torch.cat([t, t], 1)[:, :m]
    yield t.t().contiguous().t()
    yield torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(n, m)
    yield t[:1].expand(n, m)


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("T", [1, 5])
def test_inputs_of_any_layout(which, T):
    args = _tensors(T, grad=False)
    for i, v in enumerate(_views(args[which])):
        a = [t.clone().requires_grad_() for t in args]
        a[which] = v.detach().requires_grad_()
        b = [t.detach().contiguous().requires_grad_() for t in a]
        y, z = layers.gated_ffn(Owner(), *a), _plain(*b)
        assert torch.allclose(y, z), i
        got, want = torch.autograd.grad(y.square().sum(), a), torch.autograd.grad(z.square().sum(), b)
        assert all(torch.allclose(g, w) for g, w in zip(got, want)), i
        with torch.no_grad():
            assert torch.equal(layers.gated_ffn(Owner(), *a), y)


def test_more_dimensions_and_views_of_them():
    args = _tensors(6)
    x = args[0].detach().view(2, 3, 8)
    for v in (x, x.transpose(0, 1), torch.cat([x, x[..., :2]], -1)[..., :8], x[:0], x[0, 0]):
        y = layers.gated_ffn(Owner(), v, *args[1:])
        assert y.shape == v.shape and torch.allclose(y, _plain(v.reshape(-1, 8), *args[1:]).view(v.shape))


# -- norm with rotation: one of the two tensors -------------------------------------------------
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("gains", [False, True])
def test_norm_of_queries_or_keys_alone(which, gains):
    q, k, cos, sin, pos, gq, gk = _qk()
    x, g = (q, gq) if which == 0 else (k, gk)
    pair = [None, None]
    pair[which] = x
    gain = [None, None]
    if gains:
        gain[which] = g
    out = layers.qk_norm_rope(Owner(), *pair, cos, sin, pos, *gain)
    assert out[1 - which] is None
    w = torch.randn_like(x)
    leaves = (x, g) if gains else (x,)
    got = torch.autograd.grad((out[which] * w).sum(), leaves)
    want = torch.autograd.grad(((x * g if gains else x) * w).sum(), leaves)
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


def test_norm_with_one_result_unused_and_transposed_gradients():
    q, k, cos, sin, pos, gq, gk = _qk()
    a, b = layers.qk_norm_rope(Owner(), q, k, cos, sin, pos, gq, gk)
    got = torch.autograd.grad((a.transpose(1, 2).contiguous() ** 2).sum(), (q, k, gq, gk))
    want = torch.autograd.grad(((q * gq) ** 2).sum(), (q, gq))
    assert torch.allclose(got[0], want[0]) and torch.allclose(got[2], want[1])
    assert not got[1].any() and not got[3].any()
