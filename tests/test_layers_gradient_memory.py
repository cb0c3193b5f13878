"""The gradients of a norm's two addends are tensors of their own, whatever stands between the norm and the leaves: autograd keeps
what reaches a leaf without a copy, so a shared one would take in-place work on either (a second backward pass, clipping) twice."""
import pytest
import torch

from paper_2505_23725_b200 import layers
from test_decoder_operators_host import Owner, rand

PAIRS = {
    "leaves": lambda a, b: (a, b),
    "views": lambda a, b: (a.view(6, 8), b.view(6, 8)),
    "views of three dimensions": lambda a, b: (a.view(2, 3, 8), b.view(2, 3, 8)),
    "a leaf and a view": lambda a, b: (a.view(6, 8), b),
    "sums with a constant": lambda a, b: (a + 1.0, b + 1.0),
    "a leaf and a sum": lambda a, b: (a, b + 1.0),
    "a sum and a view": lambda a, b: (a + 1.0, b.view(6, 8)),
    "views of one leaf": lambda a, b: (a[:3], a[3:]),
    "one tensor twice": lambda a, b: (a, a),
}


def plain(x, r):
    h = x + r
    mean = h.mean(-1, keepdim=True)
    return (h - mean) * ((h - mean).square().mean(-1, keepdim=True) + 1e-6).rsqrt(), h


def loss(norm, pair, leaves, i):
    y, h = norm(*PAIRS[pair](*leaves))
    w = torch.linspace(-1, 1, y.numel(), dtype=y.dtype).view(y.shape) * (i + 1)
    return (y * w).sum() + (h * h).sum()


def own(x, r):
    return layers.layer_norm(Owner(), x, residual=r)


def accumulated(pair, leaves, passes):
    for i in range(passes):
        loss(own, pair, leaves, i).backward()
    return [t.grad for t in leaves]


def expected(pair, leaves, passes):
    """Each pass's gradients on their own, added up here (accumulated in .grad, torch's own sum of two views shares memory too)."""
    each = [torch.autograd.grad(loss(plain, pair, leaves, i), leaves, allow_unused=True) for i in range(passes)]
    return [None if g[0] is None else sum(t.clone() for t in g) for g in zip(*each)]


@pytest.mark.parametrize("pair", PAIRS)
def test_two_backward_passes_add_up(pair):
    torch.manual_seed(0)
    leaves = [rand(6, 8), rand(6, 8)]
    want = expected(pair, leaves, 2)
    got = accumulated(pair, leaves, 2)
    if got[0] is not None and got[1] is not None:
        assert got[0].untyped_storage().data_ptr() != got[1].untyped_storage().data_ptr()
    for a, b in zip(got, want):
        assert (a is None) == (b is None)
        assert a is None or torch.allclose(a, b, rtol=1e-10, atol=1e-12)


def test_in_place_work_on_one_gradient_leaves_the_other():
    torch.manual_seed(1)
    ga, gb = accumulated("views", [rand(6, 8), rand(6, 8)], 1)
    before = gb.clone()
    ga.mul_(2.0)
    assert torch.equal(gb, before)


def test_gradients_that_are_asked_for_are_tensors_of_their_own():
    a, b = rand(6, 8), rand(6, 8)
    x, r = a * 2.0, b * 3.0
    y, h = layers.layer_norm(Owner(), x, residual=r)
    gx, gr = torch.autograd.grad(y.square().sum() + h.sum(), (x, r))
    assert torch.equal(gx, gr) and gx.data_ptr() != gr.data_ptr()


def test_one_addend_without_a_gradient():
    for i in range(2):
        x, r = rand(6, 8, grad=i == 0), rand(6, 8, grad=i == 1)
        y, h = layers.layer_norm(Owner(), x, residual=r)
        (y.sum() + (h * h).sum()).backward()
        assert (x.grad is not None, r.grad is not None) == (i == 0, i == 1)
