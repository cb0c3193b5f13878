"""Queries with a single key: the weight is one and nothing flows into the scores, so their gradients are zero, not nearly zero."""
import pytest
import torch

from paper_2505_23725_b200 import binding
from test_gpu_attention import inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.sync_status()
    c.close()


@pytest.mark.parametrize("hq,hk,D", [(16, 2, 64), (5, 5, 112), (8, 2, 128), (3, 1, 8)])
def test_sequences_of_one_token_have_no_gradient_of_q_and_k(ctx, hq, hk, D):
    for n in (1, 3, 200):
        q, k, v, do = inputs([1] * n, 2, hq, hk, D, seed=n, spread=3.0)
        seq = binding.Sequences(ctx, [1] * n, tokens=n + 2)
        o, lse = ctx.causal_attention(q, k, v, seq)
        dq, dk, dv = ctx.causal_attention_backward(do, q, k, v, o, lse, seq)
        assert not dq.any() and not dk.any()
        # one term a query head, added in float32, rounded once; the weight as an operand of bf16 is one
        want = do[:n].double().view(n, hk, hq // hk, D).sum(2)
        size = do[:n].double().abs().view(n, hk, hq // hk, D).sum(2)
        assert ((dv[:n].double() - want).abs() <= 2.0 ** -8 * want.abs() + hq // hk * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("D", [64, 128])
def test_first_tokens_of_longer_sequences(ctx, D):
    lengths = [2, 127, 1, 128, 129, 300, 1]
    q, k, v, do = inputs(lengths, 0, 4, 2, D, seed=3)
    _, _, dq, _, _ = run(ctx, q, k, v, do, lengths)
    # (beyond 128 tokens all rows but those of the first tile take delta from o as it was rounded; the first query's tile has one key tile)
    first = torch.tensor([sum(lengths[:i]) for i in range(len(lengths))], device="cuda")
    assert not dq[first].any()


def test_values_that_are_not_finite_still_show(ctx):
    q, k, v, do = inputs([1, 1], 0, 2, 1, 64, seed=5)
    seq = binding.Sequences(ctx, [1, 1])
    o, lse = ctx.causal_attention(q, k, v, seq)
    do = do.clone()
    do[1, 0, 3] = float("nan")
    dq, dk, dv = ctx.causal_attention_backward(do, q, k, v, o, lse, seq)
    assert not dq[0].any() and not dk[0].any() and torch.isfinite(dv[0].float()).all()
    assert torch.isnan(dq[1, 0].float()).all() and torch.isnan(dk[1].float()).all() and torch.isnan(dv[1, 0, 3].float())
