"""Table gradients of batches whose sort takes one, two and three merges, and of tokens that fill hundreds of chunks, against 64 bits.

Tolerance: an entry passes at most 16 additions in a chunk, n / 128 in a warp of the join (n: tokens of the row, 16 to a chunk, 8 warps), 8 for
the warps, the scaling, and one rounding: (16 + n / 128 + 9) U32 of the magnitudes' sum."""
import pytest
import torch

from paper_2505_23725_b200 import binding
from test_gpu_norm_embedding import BF16, F32, U32, rand, rounding, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.sync_status()
    c.close()


def gradient(ctx, ids, V, d, dtype, dout_type, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dout = rand(g, ids.numel(), d, dtype=dout_type)
    got = ctx.embedding_backward(dout, ids, V, scale=0.75, dtype=dtype)
    ref = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, ids, dout.double()) * 0.75
    size = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, ids, dout.double().abs()) * 0.75
    n = torch.bincount(ids, minlength=V).double()[:, None]
    within(got, ref, (16 + n / 128 + 9) * U32 * size + rounding(dtype) * ref.abs(), "gradient")
    assert torch.equal(got, ctx.embedding_backward(dout, ids, V, scale=0.75, dtype=dtype))


@pytest.mark.parametrize("T", [511, 512, 513, 4095, 4096, 4097, 4609, 32767, 32768, 32769, 36900, 70001, 262145])
@pytest.mark.parametrize("kind", ["any", "rising", "falling"])
def test_batches_around_the_blocks_of_the_sort(ctx, T, kind):
    g = torch.Generator(device="cuda").manual_seed(T)
    V = 5000
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind != "any":
        ids = ids.sort(descending=kind == "falling")[0]
    gradient(ctx, ids, V, 8, F32, BF16, T)


@pytest.mark.parametrize("T,V,d,dtype", [(100003, 5, 40, F32), (4200, 3, 257, BF16), (300000, 2, 8, F32), (8200, 1, 24, BF16)])
@pytest.mark.parametrize("share", [1.0, 0.9])
def test_a_token_that_fills_a_batch(ctx, T, V, d, dtype, share):
    """Its row is hundreds to thousands of chunks, at the sorted order's beginning or its end."""
    g = torch.Generator(device="cuda").manual_seed(d)
    for row in {0, V - 1}:
        ids = torch.where(torch.rand(T, generator=g, device="cuda") < share, row, torch.randint(0, V, (T,), generator=g, device="cuda"))
        gradient(ctx, ids, V, d, dtype, BF16, T + row)


@pytest.mark.parametrize("V,d,dtype", [(4000, 771, F32), (1, 2048, BF16), (33, 1025, F32), (640, 1500, BF16), (31, 5000, F32), (70000, 260, F32)])
def test_rows_without_tokens_are_zero(ctx, V, d, dtype):
    """Over memory that held other values."""
    g = torch.Generator(device="cuda").manual_seed(V)
    for T in (1, 60):
        torch.full((V, d), 7.0, dtype=dtype, device="cuda")
        gradient(ctx, torch.randint(0, V, (T,), generator=g, device="cuda"), V, d, dtype, F32, T)
