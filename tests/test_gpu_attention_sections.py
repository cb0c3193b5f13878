"""Causal attention over batches whose heads do not fit into L2 together: units come in sections of heads, the last one narrower than the
others.  Against the definition in 64 bits (tolerances of test_gpu_attention.py)."""
import pytest
import torch

from paper_2505_23725_b200 import binding
from test_gpu_attention import inputs, run

pytestmark = pytest.mark.gpu

MB32 = 32 << 20


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.sync_status()
    c.close()


def widths(tokens, hk, group, D, back):
    """Key heads of the sections: as many as 32 MB of keys and values hold (in the backward pass queries and gradients too)."""
    some = max(1, min(hk, MB32 // (tokens * D * 4 * (1 + group if back else 1))))
    return [min(some, hk - i) for i in range(0, hk, some)]


CASES = [
    # count and length of sequences, key heads, group: the key heads of the sections forward and backward
    (46, 180, 11, 1, [7, 4], [3, 3, 3, 2]),
    (40, 200, 7, 3, [7], [2, 2, 2, 1]),
    (60, 200, 7, 2, [5, 2], [1] * 7),
]


@pytest.mark.parametrize("n,length,hk,group,forward,backward", CASES)
def test_sections_with_a_remainder(ctx, n, length, hk, group, forward, backward):
    lengths = [length + (i * 37) % 60 - 30 for i in range(n)]
    T = sum(lengths) + 5
    assert (widths(T, hk, group, 128, False), widths(T, hk, group, 128, True)) == (forward, backward), T
    q, k, v, do = inputs(lengths, 5, hk * group, hk, 128, "fused", seed=n)
    run(ctx, q, k, v, do, lengths)
