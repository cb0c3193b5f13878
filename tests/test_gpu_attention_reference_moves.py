"""Causal attention where the score that a row's weights refer to moves: the sums so far are rescaled in tensor memory, each half of
the columns by another warp, before the next product adds to all of them.  Against the definition in 64 bits, with the
tolerances of test_gpu_attention.py: a rescaling is one exponential and one product more (2^-21 of a sum at most, the same for numerator and total), far inside
the 2^-6 of a bf16 rounding that is allowed there."""
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


def rising(lengths, hq, hk, D, top, seed):
    """Keys that grow along every sequence: a row's largest score moves by more than the logarithm of the threshold from tile to tile."""
    q, k, v, do = inputs(lengths, 0, hq, hk, D, seed=seed)
    size = torch.cat([torch.linspace(0.1, top, n, device="cuda") for n in lengths])
    return q, (k.float() * size[:, None, None]).to(torch.bfloat16), v, do


@pytest.mark.parametrize("D", [128, 112, 96, 80, 72, 64, 24])
def test_growing_maximum(ctx, D):
    lengths = [900, 129, 300]
    run(ctx, *rising(lengths, 2, 2, D, 8.0, 5), lengths, scale=0.5)


@pytest.mark.parametrize("D", [128, 96])
@pytest.mark.parametrize("scale,spread", [(0.125, 6.0), (1.0, 2.0)])
def test_sharp_weights(ctx, D, scale, spread):
    q, k, v, do = inputs([700, 130], 0, 3, 1, D, spread=spread, seed=4)
    run(ctx, q, k, v, do, [700, 130], scale=scale)


def test_rows_that_move_beside_rows_that_do_not(ctx):
    """Every third query is small, so that its row's weights stay by its first reference."""
    lengths = [1000]
    q, k, v, do = rising(lengths, 2, 1, 128, 8.0, 6)
    q = q.clone()
    q[::3] *= 2.0 ** -6
    run(ctx, q, k, v, do, lengths, scale=0.5)


def test_long_rows_whose_reference_moves_at_every_tile_come_out_the_same_every_time(ctx):
    """32 key tiles, all multiprocessors at work: the same bits in every run, and the definition's values."""
    lengths = [4096, 2000]
    q, k, v, do = rising(lengths, 8, 2, 128, 36.0, 7)
    first = run(ctx, q, k, v, do, lengths, scale=0.5)[:2]
    seq = binding.Sequences(ctx, lengths)
    for _ in range(50):
        assert all(torch.equal(a, b) for a, b in zip(ctx.causal_attention(q, k, v, seq, scale=0.5), first))
