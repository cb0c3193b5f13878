"""The forms of the operators' kernels that real training sizes take, against the definitions in 64 bits on the GPU.

The shapes of the other tests are small: few tokens, at most a tile per worker, a step of staged heads per token.  Here
  feed-forward   every product on 256 x 256 tiles, more tiles than there are CTA pairs (a pair's second tile: the other accumulator,
                 its phases, the pipeline carried over), more than the eight tile rows that are worked through together, two operand pairs (dX)
  norm           more tokens than there can be warps, so that a token's heads all go to one warp, in several staged steps
and the sizes are asserted to do so.  Tolerances: those of test_gpu_operators.py (derived there)."""
import pytest

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    from paper_2505_23725_b200 import binding
    c = binding.Context("cuda:0")
    yield c
    c.close()


def _within(got, ref, bound, what):
    err = (got.double() - ref).abs()
    ok = err <= bound + 1e-30
    assert bool(ok.all()), f"{what}: {int((~ok).sum())} of {ref.numel()} off; worst {float((err / (bound + 1e-30)).max()):.2f} of the bound"


# ------------------------------------------------------------------------------------------------
# feed-forward
# ------------------------------------------------------------------------------------------------
FFN_SHAPES = [(4100, 1032, 1160), (20001, 136, 264), (2577, 1544, 2056), (2049, 2304, 2312)]


def _activation(g, act):
    import torch
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    k, c = (2 / torch.pi) ** 0.5, 0.044715
    th = torch.tanh(k * (g + c * g ** 3))
    return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * k * (1 + 3 * c * g * g)


def _ffn_inputs(T, d, F):
    import torch
    torch.manual_seed(T + d + F)
    bf = torch.bfloat16
    return ((torch.randn(T, d, device="cuda")).to(bf), (torch.randn(d, F, device="cuda") * d ** -0.5).to(bf),
            (torch.randn(d, F, device="cuda") * d ** -0.5).to(bf), (torch.randn(F, d, device="cuda") * F ** -0.5).to(bf),
            torch.randn(T, d, device="cuda").to(bf))


def _check_ffn(ctx, x, w1, w3, w2, dy, act):
    y, (g, u, h) = ctx.gated_ffn(x, w1, w3, w2, activation=act)
    grads = ctx.gated_ffn_backward(dy, x, w1, w3, w2, (g, u, h), activation=act)
    ctx.sync_status()
    X, W1, W3, W2, DY = (t.double() for t in (x, w1, w3, w2, dy))
    (T, d), F = X.shape, W1.shape[1]
    e = 2.0 ** -23
    G, U = X @ W1, X @ W3
    dG, dU = d * e * (X.abs() @ W1.abs()), d * e * (X.abs() @ W3.abs())
    _within(g, G, dG + U16 * G.abs(), "g")
    _within(u, U, dU + U16 * U.abs(), "u")
    value, _ = _activation(G, act)
    H = value * U
    dH = 1.2 * dG * U.abs() + dU * value.abs() + 1.2 * dG * dU + 16 * U32 * (G * U).abs()
    _within(h, H, dH + U16 * (H.abs() + dH), "h")
    del G, U, H, dG, dU, dH, value
    Gr, Ur, Hr = g.double(), u.double(), h.double()
    Y = Hr @ W2
    _within(y, Y, F * e * (Hr.abs() @ W2.abs()) + U16 * Y.abs() * 1.01, "y")
    del Y
    value, slope = _activation(Gr, act)
    DH, dDH = DY @ W2.T, d * e * (DY.abs() @ W2.T.abs())
    DG, DU = DH * Ur * slope, DH * value
    eG = dDH * (Ur * slope).abs() + 32 * U32 * (DH * Ur).abs() * (1 + Gr.abs()) + U16 * DG.abs() * 1.01
    eU = dDH * value.abs() + 32 * U32 * (DH * Gr).abs() + U16 * DU.abs() * 1.01
    del DH, dDH, value, slope, Gr, Ur
    aG, aU = DG.abs() + eG, DU.abs() + eU
    for name, got, ref, b in (
            ("dx", grads[0], lambda: DG @ W1.T + DU @ W3.T,
             lambda: eG @ W1.T.abs() + eU @ W3.T.abs() + 2 * F * e * (aG @ W1.T.abs() + aU @ W3.T.abs())),
            ("dw1", grads[1], lambda: X.T @ DG, lambda: X.T.abs() @ (eG + T * e * aG)),
            ("dw3", grads[2], lambda: X.T @ DU, lambda: X.T.abs() @ (eU + T * e * aU)),
            ("dw2", grads[3], lambda: Hr.T @ DY, lambda: T * e * (Hr.T.abs() @ DY.abs()))):
        ref, b = ref(), b()
        _within(got, ref, b + U16 * (ref.abs() + b), name)
        rel = float((got.double() - ref).norm() / ref.norm())
        assert rel < 4e-3, f"{name}: {rel:.2e}"
    return (y, g, u, h, *grads)


def _all_large(T, d, F):
    import torch
    from paper_2505_23725_b200 import binding
    n_sms = torch.cuda.get_device_properties(0).multi_processor_count
    forms, tiles = binding.ffn_forms(T, d, F, n_sms)
    assert forms == {"gate", "y", "gate_back", "dx"}, (T, d, F, forms)
    assert min(tiles) > n_sms // 2 and T > 8 * 256, (T, d, F, tiles)


@pytest.mark.parametrize("shape", FFN_SHAPES, ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_feed_forward_on_large_tiles(ctx, shape, act):
    import torch
    _all_large(*shape)
    x, w1, w3, w2, dy = _ffn_inputs(*shape)
    first = _check_ffn(ctx, x, w1, w3, w2, dy, act)
    y, saved = ctx.gated_ffn(x, w1, w3, w2, activation=act)
    again = (y, *saved, *ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved, activation=act))
    assert all(torch.equal(a, b) for a, b in zip(first, again))          # sums in a fixed order
    assert torch.equal(ctx.gated_ffn(x, w1, w3, w2, activation=act, save=False)[0], y)


def test_feed_forward_on_large_tiles_strided(ctx):
    """Activations and weights as parts of wider matrices, rows 16 but not 32 bytes apart among them."""
    import torch
    T, d, F = 4100, 1032, 1160
    _all_large(T, d, F)
    x, w1, w3, w2, dy = _ffn_inputs(T, d, F)
    def part(t, before, after):
        wide = torch.zeros(t.shape[0], before + t.shape[1] + after, dtype=t.dtype, device="cuda")
        wide[:, before:before + t.shape[1]] = t
        return wide[:, before:before + t.shape[1]]
    both = torch.cat([w1, w3], 1)
    args = part(x, 8, 16), both[:, :F], both[:, F:], part(w2, 24, 8)
    dys = part(dy, 16, 0)
    y, saved = ctx.gated_ffn(*args)
    got = (y, *saved, *ctx.gated_ffn_backward(dys, *args, saved))
    y, saved = ctx.gated_ffn(x, w1, w3, w2)
    want = (y, *saved, *ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ctx.sync_status()


def test_each_gradient_alone(ctx):
    """Gradients that are not wanted are NULL at the C entry point: the others are the same bits, on either form."""
    import torch
    from paper_2505_23725_b200 import binding
    for T, d, F in ((4100, 1032, 1160), (200, 1024, 392)):
        x, w1, w3, w2, dy = _ffn_inputs(T, d, F)
        y, (g, u, h) = ctx.gated_ffn(x, w1, w3, w2)
        want = ctx.gated_ffn_backward(dy, x, w1, w3, w2, (g, u, h))
        a = binding._FFN_PACK(T, d, F, d, F, F, d, x.data_ptr(), w1.data_ptr(), w3.data_ptr(), w2.data_ptr(), 0, 0)
        for keep in range(16):
            out = [torch.full_like(t, 7.0) for t in want]
            dg, du = torch.empty_like(g), torch.empty_like(u)
            ptrs = [t.data_ptr() if keep >> i & 1 else None for i, t in enumerate(out)]
            assert ctx.lib.muloco_gated_ffn_backward(ctx.ctx, a, dy.data_ptr(), d, g.data_ptr(), u.data_ptr(), h.data_ptr(),
                                                     dg.data_ptr(), du.data_ptr(), *ptrs) == binding.OK
            for i, t in enumerate(out):
                assert torch.equal(t, want[i]) if keep >> i & 1 else bool((t == 7.0).all()), (T, keep, i)
    ctx.sync_status()


# ------------------------------------------------------------------------------------------------
# norm with rotation
# ------------------------------------------------------------------------------------------------
MAX_WARPS = 148 * 16 * 4                     # more than any launch has (16 blocks of four warps an SM)
QK_CASES = [
    # heads of q and k, head size, rotated part, interleaved
    (19, 5, 128, 128, False), (16, 16, 128, 64, True), (13, 3, 64, 32, True), (9, 2, 100, 52, True), (7, 1, 508, 508, False),
    (5, 0, 256, 256, False), (0, 11, 96, 96, True), (6, 3, 90, 90, False), (4, 2, 512, 512, True),
]


def _turn(x, cos, sin, il, sign=1.0):
    import torch
    r = cos.shape[-1]
    c, s = cos[:, None], sign * sin[:, None]
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if il else (x[..., :r], x[..., r:2 * r])
    y, z = a * c - b * s, b * c + a * s
    t = torch.stack((y, z), -1).flatten(-2) if il else torch.cat((y, z), -1)
    return torch.cat((t, x[..., 2 * r:]), -1)


def _pairs(x, r, il):
    """|first| + |second| of every entry's pair, |x| of the entries that are not turned."""
    import torch
    x = x.abs()
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if il else (x[..., :r], x[..., r:2 * r])
    s = a + b
    t = torch.stack((s, s), -1).flatten(-2) if il else torch.cat((s, s), -1)
    return torch.cat((t, x[..., 2 * r:]), -1)


@pytest.mark.parametrize("case", QK_CASES, ids=str)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norm_in_several_steps_per_token(ctx, case, dtype):
    import torch
    hq, hk, D, rot, il = case
    T, dt = MAX_WARPS + 533, getattr(torch, dtype)
    torch.manual_seed(D + hq)
    low = U16 if dt == torch.bfloat16 else 0.0
    eps = 1e-5
    q, k, dq, dk = (torch.randn(T, h, D, device="cuda").to(dt) if h else None for h in (hq, hk, hq, hk))
    ang = torch.randn(T + 9, rot // 2, device="cuda", dtype=torch.float64) * 3
    cos, sin = ang.cos().float(), ang.sin().float()
    pos = torch.randint(0, T + 9, (T,), device="cuda")
    gq, gk = (1 + 0.3 * torch.randn(D, device="cuda") for _ in range(2))
    out = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk, eps, il)
    back = ctx.qk_norm_rope_backward(dq, dk, q, k, cos, sin, pos, gq, gk, eps, il)
    again = ctx.qk_norm_rope_backward(dq, dk, q, k, cos, sin, pos, gq, gk, eps, il)
    ctx.sync_status()
    for a, b in zip(back, again):
        assert (a is None and b is None) or torch.equal(a, b)
    c, s = cos.double()[pos], sin.double()[pos]
    e32 = float(torch.tensor(eps))
    for x, y, dy, dx, g, dg in ((q, out[0], dq, back[0], gq, back[2]), (k, out[1], dk, back[1], gk, back[3])):
        if x is None:
            assert y is None and dx is None and dg is None
            continue
        X, DY, G = x.double(), dy.double(), g.double()
        r = 1 / (X.square().mean(-1, keepdim=True) + e32).sqrt()
        ref = _turn(X * r * G, c, s, il)
        _within(y, ref, 32 * U32 * _pairs(X * r * G, rot // 2, il) + low * ref.abs(), "forward")
        n, dn, mag = X * r, _turn(DY, c, s, il, -1.0), _pairs(DY, rot // 2, il)
        ref = r * (G * dn - n * (G * dn * n).mean(-1, keepdim=True))
        mean = (G.abs() * mag * n.abs()).mean(-1, keepdim=True)
        _within(dx, ref, 64 * U32 * r * (G.abs() * mag + n.abs() * mean) + low * ref.abs(), "backward")
        _within(dg, (dn * n).sum((0, 1)), 128 * U32 * (mag * n.abs()).sum((0, 1)), "gain")
