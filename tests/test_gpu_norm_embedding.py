"""Norm over the last dimension and embedding lookup on the GPU, against their definitions in 64 bits.

Tolerances, per element (U16 = 2^-8, U32 = 2^-24: a rounding to bf16, to float32).
  norm: entries of y pass a sum of d terms (tree of lanes and a chain of at most 32 in a lane: 64 roundings), a root, a quotient, and
    four operations: 80 U32 of the magnitudes (|h| + |mean|) rstd |weight| + |bias|, the mean's own error (64 U32 of
    mean |h|) among them, and a bf16 rounding.  rstd: 80 U32 and the mean's share.
    dx = rstd (e - n c1 - c2) + dh: 128 U32 of the magnitudes of its terms, with c1 and c2 by the mean of magnitudes.
    dweight, dbias: sums over tokens, T / 296 of them in a chain: (T / 296 + 40) U32 of the magnitudes' sum, and those of n.
  embedding: exact product, one rounding.  Gradient: at most 64 terms, or pieces of 64, in a chain: (64 + T / 512 + 8) U32 of the
    magnitudes' sum, and one rounding."""
import pytest
import torch

from paper_2505_23725_b200 import binding

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.close()


def rand(g, *shape, dtype=F32, s=1.0, at=0.0):
    return (torch.randn(*shape, generator=g, device="cuda") * s + at).to(dtype)


def within(got, ref, tol, name):
    got = got.double()
    assert got.shape == ref.shape, name
    assert torch.isfinite(got).all(), name
    bad = (got - ref).abs() > tol + 1e-30
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} beyond the tolerance, " \
                          f"worst {((got - ref).abs() / (tol + 1e-30)).max():.2f} of it"


def rounding(dtype):
    return U16 if dtype == BF16 else U32


NORM = [
    # tokens, d, dtype, center, weight, bias, residual
    (1, 1, F32, True, True, True, True),
    (3, 7, BF16, True, True, True, True),
    (1, 768, BF16, False, True, False, True),
    (33, 256, BF16, True, True, True, False),
    (65, 257, F32, False, True, False, False),
    (300, 771, F32, True, True, True, True),
    (4099, 768, BF16, False, True, False, True),
    (130, 1024, F32, True, False, True, False),
    (129, 1032, BF16, True, True, False, True),
    (77, 2048, BF16, True, True, True, True),
    (50, 2050, BF16, False, True, False, False),
    (19, 4096, F32, True, True, True, True),
    (9, 8192, BF16, False, True, False, True),
    (5, 8200, BF16, True, True, True, True),
    (3, 32768, F32, True, True, True, False),
    (2, 32767, BF16, False, False, False, True),
]


@pytest.mark.parametrize("T,d,dtype,center,weight,bias,residual", NORM, ids=lambda x: str(x).replace("torch.", ""))
def test_norm(ctx, T, d, dtype, center, weight, bias, residual):
    g = torch.Generator(device="cuda").manual_seed(T * 1000 + d)
    x = rand(g, T, d, dtype=dtype, s=2.0, at=0.7)
    w = rand(g, d, s=0.3, at=1.0) if weight else None
    b = rand(g, d, s=0.3) if bias else None
    r = rand(g, T, d, dtype=dtype) if residual else None
    eps = 2.0 ** -18
    y, h, rstd, mean = ctx.layer_norm(x, w, b, r, eps=eps, center=center)
    W = w.double() if weight else torch.ones(d, dtype=torch.float64, device="cuda")
    B = b.double() if bias else torch.zeros(d, dtype=torch.float64, device="cuda")
    H = x.double() + r.double() if residual else x.double()
    m = H.mean(1, keepdim=True) if center else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
    off = 64 * U32 * H.abs().mean(1, keepdim=True) if center else 0.0 * m       # of the mean
    R = (((H - m) ** 2).mean(1, keepdim=True) + eps) ** -0.5
    # an entry's difference from the mean is off by `off` and its own roundings, and the spread by as much in the mean square
    relative = 80 * U32 + 2 * ((off + U32 * (H.abs() + m.abs())).square().mean(1, keepdim=True)).sqrt() * R
    Y = (H - m) * R * W + B
    within(rstd, R[:, 0], (relative * R)[:, 0], "rstd")
    if center:
        within(mean, m[:, 0], off[:, 0] + U32 * m.abs()[:, 0], "mean")
    if residual:
        within(h, H, rounding(dtype) * H.abs(), "h")
    else:
        assert h is x
    tol_y = relative * (H - m).abs() * R * W.abs() + (off + U32 * (H.abs() + m.abs())) * R * W.abs() + 4 * U32 * (Y.abs() + B.abs())
    within(y, Y, tol_y + rounding(dtype) * Y.abs(), "y")

    # backward, from the rounded h and the definition's statistics
    dy = rand(g, T, d, dtype=dtype)
    dh = rand(g, T, d, dtype=dtype) if residual else None
    Hr = h.double()
    rs, mu = R[:, 0].float(), m[:, 0].float()
    dx, dw, db = ctx.layer_norm_backward(dy, h, rs, mu if center else None, weight=w, dh=dh, bias=bias)
    Rr, mr = rs.double()[:, None], mu.double()[:, None]
    N = (Hr - mr) * Rr
    E = dy.double() * W
    c1, c2 = (E * N).mean(1, keepdim=True), E.mean(1, keepdim=True) if center else 0.0 * m
    D = dh.double() if residual else torch.zeros_like(E)
    DX = Rr * (E - N * c1 - c2) + D
    size = Rr * (E.abs() + N.abs() * (E * N).abs().mean(1, keepdim=True) + (E.abs().mean(1, keepdim=True) if center else 0.0)) + D.abs()
    # (n = (h - mean) rstd is off by a rounding of h - mean, whose terms may cancel)
    nerr = 4 * U32 * (Hr.abs() + mr.abs()) * Rr
    size_n = Rr * (nerr * c1.abs() + N.abs() * (E.abs() * nerr).mean(1, keepdim=True))
    within(dx, DX, 128 * U32 * size + size_n + rounding(dtype) * DX.abs(), "dx")
    chain = (T / 296 + 40) * U32
    if weight:
        within(dw, (dy.double() * N).sum(0), chain * (dy.double() * N).abs().sum(0) + (dy.double().abs() * nerr).sum(0), "dweight")
    else:
        assert dw is None
    if bias:
        within(db, dy.double().sum(0), chain * dy.double().abs().sum(0), "dbias")
    else:
        assert db is None
    ctx.sync_status()


def test_norm_of_views_and_constant_rows(ctx):
    """Rows of a wider matrix at odd offsets; a row without spread gives the bias; a row far from zero keeps its digits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    wide = rand(g, 40, 700)
    for first, d in ((0, 512), (4, 512), (3, 512), (1, 333)):
        x = wide[:, first:first + d]
        y, _, rstd, mean = ctx.layer_norm(x, eps=1e-6)
        y2, _, rstd2, mean2 = ctx.layer_norm(x.contiguous(), eps=1e-6)
        within(y, y2.double(), 1e-6 * (1 + y2.abs().double()), "view")
        dx, _, _ = ctx.layer_norm_backward(wide[:, first + 1:first + 1 + d], x, rstd, mean)
        dx2, _, _ = ctx.layer_norm_backward(wide[:, first + 1:first + 1 + d].contiguous(), x.contiguous(), rstd, mean)
        within(dx, dx2.double(), 1e-6 * (1 + dx2.abs().double()), "view, backward")
    b = rand(g, 96)
    y, _, rstd, _ = ctx.layer_norm(torch.full((3, 96), 5.0, device="cuda"), bias=b, eps=1e-4)
    assert torch.equal(y, b.expand(3, 96)) and torch.allclose(rstd, torch.full((3,), 100.0, device="cuda"), rtol=1e-6)
    x = 4096.0 + torch.randint(-8, 9, (5, 640), generator=g, device="cuda").float()      # sums of exact values
    y, _, _, _ = ctx.layer_norm(x, eps=0.0)
    X = x.double()
    within(y, (X - X.mean(1, keepdim=True)) / X.var(1, unbiased=False, keepdim=True).sqrt(), torch.full_like(X, 1e-3), "far from zero")


EMB = [
    # tokens, rows, d, dtype of the table and its gradient, of dout, kind of ids
    (1, 1, 1, F32, F32, "any"),
    (1, 5, 768, BF16, BF16, "any"),
    (7, 100, 48, F32, BF16, "any"),
    (64, 33, 256, BF16, BF16, "one"),
    (65, 32, 264, F32, BF16, "one"),
    (130, 64, 257, BF16, F32, "one"),
    (1000, 31, 100, F32, F32, "any"),
    (2048, 500, 64, F32, BF16, "any"),
    (2049, 500, 72, F32, BF16, "few"),
    (5000, 7, 520, BF16, BF16, "few"),
    (16385, 1000, 40, F32, F32, "few"),
    (20000, 32000, 16, BF16, BF16, "any"),
    (140001, 300, 24, F32, BF16, "few"),
]


@pytest.mark.parametrize("T,V,d,dtype,dout_type,kind", EMB, ids=lambda x: str(x).replace("torch.", ""))
def test_embedding(ctx, T, V, d, dtype, dout_type, kind):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind == "one":
        ids[:] = V - 1
    if kind == "few":                        # most tokens are one of three
        ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.8, ids % 3 * (V // 3), ids)
    table = rand(g, V, d, dtype=dtype)
    out = ctx.embedding(ids, table, scale=0.3)
    s = torch.tensor(0.3, dtype=F32).double().item()
    ref = s * table.double()[ids]
    within(out, ref, (rounding(dtype) + U32) * ref.abs(), "embedding")
    dout = rand(g, T, d, dtype=dout_type)
    got = ctx.embedding_backward(dout, ids, V, scale=0.3, dtype=dtype)
    ref = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, ids, dout.double()) * s
    size = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, ids, dout.double().abs()) * s
    within(got, ref, (64 + T / 512 + 8) * U32 * size + rounding(dtype) * ref.abs(), "gradient")
    unused = torch.ones(V, dtype=torch.bool, device="cuda")
    unused[ids] = False
    assert not got[unused].any()
    for _ in range(3):                       # the order of the sums is fixed
        assert torch.equal(got, ctx.embedding_backward(dout, ids, V, scale=0.3, dtype=dtype))
    ctx.sync_status()


def test_tokens_outside_the_table(ctx):
    g = torch.Generator(device="cuda").manual_seed(1)
    table, dout = rand(g, 10, 24), rand(g, 6, 24)
    ids = torch.tensor([3, -1, 9, 10, 2 ** 40, 3], device="cuda")
    out = ctx.embedding(ids, table)
    with pytest.raises(binding.MulocoError) as e:
        ctx.sync_status()
    assert e.value.status == binding.EINVAL and "outside the embedding's table" in str(e.value)
    good = torch.tensor([0, 2, 5], device="cuda")
    assert torch.equal(out[good], table[ids[good]]) and torch.isnan(out[[1, 3, 4]]).all()
    got = ctx.embedding_backward(dout, ids, 10)
    with pytest.raises(binding.MulocoError):
        ctx.sync_status()
    ref = torch.zeros(10, 24, device="cuda").index_add_(0, ids[good], dout[good])
    assert torch.allclose(got, ref, rtol=1e-6, atol=1e-6)
    # many of them, in pieces of their own
    ids = torch.full((300,), -5, device="cuda")
    ids[7] = 4
    dout = rand(g, 300, 24)
    got = ctx.embedding_backward(dout, ids, 10)
    with pytest.raises(binding.MulocoError):
        ctx.sync_status()
    assert torch.equal(got[4], dout[7]) and not got[torch.arange(10) != 4].any()


def test_no_tokens(ctx):
    z = torch.empty(0, 64, device="cuda")
    y, _, rstd, mean = ctx.layer_norm(z)
    assert y.shape == (0, 64) and rstd.shape == (0,)
    _, dw, db = ctx.layer_norm_backward(z, z, rstd, mean, weight=torch.ones(64, device="cuda"), bias=True)
    assert not dw.any() and not db.any()
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    assert ctx.embedding(ids, torch.ones(3, 64, device="cuda")).shape == (0, 64)
    assert not ctx.embedding_backward(z, ids, 3).any()
    ctx.sync_status()
