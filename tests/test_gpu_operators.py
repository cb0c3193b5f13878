"""GPU parity of the operators around the optimizer step -- AdamW lists, the norm of queries and keys with the
rotation, the gated feed-forward block -- against their float64 definitions.

Tolerances (U32 = 2^-24, U16 = 2^-8: unit roundoffs of float32 (24 bits) and bf16 (8 bits)):
  AdamW       theta, 32-bit moments: the library's 1e-6; 8-bit codes, scales and moments: bit for bit.
  norm        per entry, float32: 32 U32 (|first| + |second|) of the turned pair -- the sum of squares (a dozen roundings
              of a positive sum), the root, three products and a sum; the same and one bf16 rounding for bf16.
              dx adds up two terms, each within 32 U32 of its magnitude.  dgain: 128 U32 of the terms' magnitudes summed.
  feed-forward  a sum of n products in float32: n 2^-23 of the magnitudes' sum (the tensor cores may truncate), one
              bf16 rounding per stored tensor, and for dX, dW1, dW3 the rounding of dG and dU carried through the product."""
import numpy as np
import pytest

from helpers import assert_close_1e6
from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    from paper_2505_23725_b200 import binding
    c = binding.Context("cuda:0")
    yield c
    c.close()


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(rng, *shape, scale=1.0):
    import torch
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16).cuda()


def _within(got, ref, bound, what):
    err = np.abs(_np(got) - ref)
    ok = err <= bound + 1e-30
    assert ok.all(), f"{what}: {int((~ok).sum())} of {ref.size} off; worst {float((err / (bound + 1e-30)).max()):.2f} of the bound"


# ------------------------------------------------------------------------------------------------
# AdamW
# ------------------------------------------------------------------------------------------------
SIZES = [[1], [255, 256, 257], [3, 1000, 2049, 64 * 100, 5], [300_007]]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


def _list(ctx, sizes, bits, gdtype, copies=False, **kw):
    import torch
    from paper_2505_23725_b200 import binding
    rng = np.random.default_rng(sum(sizes) + bits)
    host = [(rng.standard_normal(n) * 0.02).astype(np.float32) for n in sizes]
    params = [torch.from_numpy(h.copy()).cuda() for h in host]
    cps = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes] if copies else None
    opt = binding.AdamW(ctx, params, state_bits=bits, grad_dtype=gdtype, copies=cps, **{**HYPER, **kw})
    return rng, host, params, cps, opt


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_adamw_32_bit_states(ctx, sizes, bf16):
    import torch
    dt = torch.bfloat16 if bf16 else torch.float32
    wd = [1.0 if i % 2 else 0.0 for i in range(len(sizes))]
    lm = [1.0 + i for i in range(len(sizes))]
    rng, host, params, cps, opt = _list(ctx, sizes, 32, dt, copies=True, wd_mult=wd, lr_mult=lm)
    m = [np.zeros(n) for n in sizes]
    v = [np.zeros(n) for n in sizes]
    theta = [h.astype(np.float64) for h in host]
    for t in range(1, 5):
        grads = [torch.from_numpy((rng.standard_normal(n) * 1e-3).astype(np.float32)).to(dt).cuda() for n in sizes]
        opt.step(grads, lr_scale=0.5)
        for i, g in enumerate(grads):
            # the bound of a step on float32 state: compare each step from the library's own state
            new, m[i], v[i] = O.adamw(theta[i], _np(g), m[i], v[i], t, 0.5 * HYPER["lr"] * lm[i], HYPER["beta1"],
                                      HYPER["beta2"], HYPER["eps"], HYPER["weight_decay"] * wd[i])
            o, n = opt.offsets[i], sizes[i]
            assert_close_1e6(_np(params[i]), new, f"theta {i} step {t}")
            assert_close_1e6(_np(opt.state1[o:o + n]), m[i], f"m {i} step {t}")
            assert_close_1e6(_np(opt.state2[o:o + n]), v[i], f"v {i} step {t}")
            assert torch.equal(cps[i], params[i].to(torch.bfloat16))
            theta[i], m[i], v[i] = _np(params[i]), _np(opt.state1[o:o + n]), _np(opt.state2[o:o + n])
    ctx.sync_status()
    assert opt.steps == 4
    opt.close()


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
def test_adamw_8_bit_states_bit_for_bit(ctx, sizes, bf16):
    import torch
    dt = torch.bfloat16 if bf16 else torch.float32
    rng, host, params, _, opt = _list(ctx, sizes, 8, dt, seed=99)
    st = [(np.zeros(-(-n // 256) * 256, np.int8), np.zeros(-(-n // 256), np.float32),
           np.zeros(-(-n // 256) * 256, np.uint8), np.zeros(-(-n // 256), np.float32)) for n in sizes]
    for t in range(1, 6):
        # scales from block to block, zeros, and in step 3 gradients so small that a block is encoded as zeros
        grads = []
        for n in sizes:
            g = (rng.standard_normal(n) * 10.0 ** rng.uniform(-6, 0, n)).astype(np.float32)
            g[rng.random(n) < 0.1] = 0.0
            grads.append(torch.from_numpy(g * np.float32(1e-30 if t == 3 and n < 300 else 1)).to(dt).cuda())
        theta = [_np(p) for p in params]
        opt.step(grads)
        m, v = opt.moments()
        for i, g in enumerate(grads):
            n, o = sizes[i], opt.offsets[i]
            nb = -(-n // 256)
            c1, s1, c2, s2, mm, root = O.adamw8(g.float().cpu().numpy(), *st[i], t, o, 99, 0.9, 0.99)
            assert np.array_equal(opt.state1[o:o + nb * 256].cpu().numpy()[:n], c1[:n]), (i, t)
            assert np.array_equal(opt.state2[o:o + nb * 256].cpu().numpy()[:n], c2[:n]), (i, t)
            assert np.array_equal(opt.scale1[o // 256:o // 256 + nb].cpu().numpy(), s1)
            assert np.array_equal(opt.scale2[o // 256:o // 256 + nb].cpu().numpy(), s2)
            b = np.arange(n) // 256
            assert np.array_equal(m[o:o + n].cpu().numpy(), c1[:n].astype(np.float32) * s1[b])
            r = c2[:n].astype(np.float32) * s2[b]
            assert np.array_equal(v[o:o + n].cpu().numpy(), r * r)
            bc1, bc2 = 1 - float(np.float32(0.9)) ** t, 1 - float(np.float32(0.99)) ** t
            lr, wd = float(np.float32(HYPER["lr"])), float(np.float32(HYPER["weight_decay"]))
            new = theta[i] - lr * (mm / bc1 / (root / np.sqrt(bc2) + float(np.float32(1e-8))) + wd * theta[i])
            assert_close_1e6(_np(params[i]), new, f"theta {i} step {t}")
            st[i] = (c1, s1, c2, s2)
    ctx.sync_status()
    opt.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_misaligned_views_equal_aligned_ones(ctx, bits):
    """Parameters, gradients and copies at odd addresses: the same bits as at aligned ones."""
    import torch
    from paper_2505_23725_b200 import binding
    n = 1030
    for dt in (torch.float32, torch.bfloat16):
        outs = []
        for off in (0, 1, 3):
            torch.manual_seed(5)
            base = torch.randn(n, device="cuda") * 0.02
            gbase = (torch.randn(n, device="cuda") * 1e-3).to(dt)
            p, g = torch.empty(n + 4, device="cuda")[off:off + n], torch.empty(n + 4, device="cuda", dtype=dt)[off:off + n]
            c = torch.empty(n + 4, device="cuda", dtype=torch.bfloat16)[off:off + n]
            p.copy_(base)
            g.copy_(gbase)
            opt = binding.AdamW(ctx, [p], grads=[g], copies=[c], state_bits=bits, seed=1, **HYPER)
            for _ in range(3):
                opt.step()
            outs.append((p.clone(), c.clone(), opt.state1.clone(), opt.state2.clone()))
            opt.close()
        for other in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    ctx.sync_status()


def test_adamw_resume_and_empty_tensors(ctx):
    import torch
    from paper_2505_23725_b200 import binding
    torch.manual_seed(1)
    p = [torch.randn(700, device="cuda"), torch.empty(0, device="cuda"), torch.randn(3, 5, device="cuda")]
    g = [torch.randn_like(x) for x in p]
    q = [x.clone() for x in p]
    a = binding.AdamW(ctx, p, grads=g, state_bits=8, seed=4, **HYPER)
    for _ in range(4):
        a.step()
    b = binding.AdamW(ctx, q, grads=g, state_bits=8, seed=4, **HYPER)
    for _ in range(2):
        b.step()
    c = binding.AdamW(ctx, q, grads=g, state_bits=8, seed=4, **HYPER)      # states and the count carried over
    for name in ("state1", "state2", "scale1", "scale2"):
        getattr(c, name).copy_(getattr(b, name))
    c.steps = b.steps
    for _ in range(2):
        c.step()
    assert all(torch.equal(x, y) for x, y in zip(p, q))
    ctx.sync_status()
    empty = binding.AdamW(ctx, [], state_bits=8, **HYPER)
    empty.step([])
    for o in (a, b, c, empty):
        o.close()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_adamw_flags_a_gradient_that_is_not_finite(ctx, bits, value):
    import torch
    from paper_2505_23725_b200 import binding
    p, g = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    g[700] = value
    opt = binding.AdamW(ctx, [p], grads=[g], state_bits=bits, **HYPER)
    opt.step()
    with pytest.raises(binding.MulocoError) as e:
        ctx.sync_status()
    assert e.value.status == binding.ENONFINITE
    # the blocks without it are untouched by it
    assert torch.isfinite(p[:512]).all() and torch.isfinite(p[768:]).all() and not torch.isfinite(p[700])
    if bits == 8:
        m, _ = opt.moments()
        assert torch.isfinite(m[:512]).all() and torch.isnan(m[512:768]).any()
    ctx.sync_status()
    opt.close()


def test_adamw_refusals(ctx):
    import torch
    from paper_2505_23725_b200 import binding
    p = [torch.zeros(10, device="cuda")]
    for kw in (dict(state_bits=16), dict(grads=[torch.zeros(9, device="cuda")]), dict(wd_mult=[1.0, 1.0]),
               dict(copies=[torch.zeros(10, device="cuda")]), dict(grad_dtype=torch.float16), dict(grads=[torch.zeros(10)])):
        with pytest.raises(ValueError):
            binding.AdamW(ctx, p, **kw)
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0)):
        with pytest.raises(binding.MulocoError) as e:
            binding.AdamW(ctx, p, **kw)
        assert e.value.status == binding.EINVAL
    opt = binding.AdamW(ctx, p)
    with pytest.raises(binding.MulocoError) as e:
        opt.step()                                             # no gradients anywhere
    assert e.value.status == binding.EINVAL and opt.steps == 0
    with pytest.raises(ValueError):
        opt.step([torch.zeros(10, device="cuda", dtype=torch.bfloat16)])
    opt.close()


# ------------------------------------------------------------------------------------------------
# norm of queries and keys with the rotation
# ------------------------------------------------------------------------------------------------
QK_CASES = [
    # tokens, heads of q and k, head size, rotated part, interleaved
    (1, 12, 12, 64, 64, False), (1, 3, 1, 128, 128, True), (5, 16, 4, 128, 64, False), (67, 5, 5, 80, 80, False),
    (33, 7, 2, 96, 32, True), (130, 2, 9, 256, 256, False), (19, 1, 1, 512, 512, False), (40, 6, 3, 90, 90, False),
    (40, 6, 3, 90, 44, True), (9, 4, 4, 2, 2, False), (300, 12, 3, 64, 0, False), (2000, 3, 2, 32, 32, True),
    (31, 0, 4, 64, 64, False), (31, 4, 0, 510, 510, True), (45, 5, 3, 236, 236, False), (45, 5, 3, 100, 52, True),
    (600, 3, 2, 508, 508, False), (77, 9, 4, 36, 12, False),
]


def _qk_inputs(case, dt, seed=0, layout="dense"):
    import torch
    T, hq, hk, D, rot, il = case
    rng = np.random.default_rng(seed + T + D)

    def heads(h, wide):
        if not h:
            return None
        x = torch.from_numpy(rng.standard_normal((T, h, D)).astype(np.float32)).to(dt).cuda()
        if layout == "dense":
            return x
        if layout == "heads first":                            # [heads, tokens, dim] in memory
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        buf = torch.zeros(T, h * D + wide, dtype=dt, device="cuda")   # rows of a wider projection, odd offsets too
        v = buf[:, wide // 2:wide // 2 + h * D].view(T, h, D)
        v.copy_(x)
        return v

    q, k = heads(hq, 16), heads(hk, 6)
    length = T + 3
    ang = rng.standard_normal((length, rot // 2)) * 3
    cos, sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    pos = torch.from_numpy(rng.integers(0, length, T)).cuda()
    gq, gk = (torch.from_numpy(1 + 0.3 * rng.standard_normal(D).astype(np.float32)).float().cuda() for _ in range(2))
    dq, dk = (torch.from_numpy(rng.standard_normal((T, h, D)).astype(np.float32)).to(dt).cuda() if h else None for h in (hq, hk))
    return q, k, cos, sin, pos, gq, gk, dq, dk


def _pair_magnitude(x, rot, il):
    """|first| + |second| of every entry's pair."""
    a, b = O._pairs(x.shape[-1], rot, il)
    m = np.abs(x).copy()
    s = m[..., a] + m[..., b]
    m[..., a], m[..., b] = s, s
    return m


def _check_qk(ctx, case, dt, layout="dense", positions=True, gains=True):
    import torch
    T, hq, hk, D, rot, il = case
    q, k, cos, sin, pos, gq, gk, dqo, dko = _qk_inputs(case, dt, layout=layout)
    if not positions:
        pos = None
    if not gains:
        gq = gk = None
    eps = 1e-5
    qo, ko = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk, eps, il)
    dq, dk, dgq, dgk = ctx.qk_norm_rope_backward(dqo, dko, q, k, cos, sin, pos, gq, gk, eps, il)
    ctx.sync_status()
    rows = _np(pos).astype(int) if pos is not None else np.arange(T)
    c, s = _np(cos)[rows], _np(sin)[rows]
    low = U16 if dt == torch.bfloat16 else 0.0
    for x, out, dy, dx, g, dg in ((q, qo, dqo, dq, gq, dgq), (k, ko, dko, dk, gk, dgk)):
        if x is None:
            assert out is None and dx is None and dg is None
            continue
        X, DY = _np(x), _np(dy)
        G = _np(g) if g is not None else np.ones(D)
        e32 = float(np.float32(eps))
        ref = O.qk_norm(X, G, c, s, e32, il)
        r = 1 / np.sqrt((X * X).mean(-1, keepdims=True) + e32)
        mag = _pair_magnitude(X * r * G, rot, il)
        _within(out, ref, 32 * U32 * mag + low * np.abs(ref), "forward")
        rdx, rdg, terms = O.qk_norm_backward(DY, X, G, c, s, e32, il)
        dn = _pair_magnitude(DY, rot, il)                      # bounds |R^T dy| entry by entry
        mean = (np.abs(G) * dn * np.abs(X) * r).mean(-1, keepdims=True)
        mag = r * (np.abs(G) * dn + np.abs(X) * r * mean)
        _within(dx, rdx, 64 * U32 * mag + low * np.abs(rdx), "backward")
        bound = (dn * np.abs(X) * r).sum((0, 1))
        _within(dg, rdg, 128 * U32 * bound, "gain")


@pytest.mark.parametrize("case", QK_CASES, ids=str)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norm_with_rotation(ctx, case, dtype):
    import torch
    _check_qk(ctx, case, getattr(torch, dtype))


@pytest.mark.parametrize("layout", ["heads first", "wide"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norm_with_rotation_strided(ctx, layout, dtype):
    import torch
    for case in (QK_CASES[2], QK_CASES[3], QK_CASES[8]):
        _check_qk(ctx, case, getattr(torch, dtype), layout=layout)


def test_norm_with_rotation_defaults(ctx):
    import torch
    _check_qk(ctx, QK_CASES[2], torch.bfloat16, positions=False, gains=False)
    _check_qk(ctx, QK_CASES[7], torch.float32, positions=False, gains=True)


def test_norm_in_place_and_repeatable(ctx):
    import torch
    case = (500, 8, 2, 128, 128, False)
    q, k, cos, sin, pos, gq, gk, dqo, dko = _qk_inputs(case, torch.bfloat16, layout="wide")
    want = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk)
    first = ctx.qk_norm_rope_backward(dqo, dko, q, k, cos, sin, pos, gq, gk)
    for _ in range(3):                                         # sums in a fixed order: the same bits
        again = ctx.qk_norm_rope_backward(dqo, dko, q, k, cos, sin, pos, gq, gk)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    got = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    ctx.sync_status()


def test_norm_of_nothing_and_of_zeros(ctx):
    import torch
    q, k, cos, sin, pos, gq, gk, dqo, dko = _qk_inputs((0, 4, 2, 64, 64, False), torch.float32)
    qo, ko = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk)
    out = ctx.qk_norm_rope_backward(dqo, dko, q, k, cos, sin, pos, gq, gk)
    ctx.sync_status()
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)
    assert not out[2].any() and not out[3].any()               # an empty sum
    q, k, cos, sin, pos, gq, gk, _, _ = _qk_inputs((6, 4, 2, 64, 64, False), torch.float32)
    q.zero_()
    qo, _ = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk, eps=1e-6)
    assert not qo.any()
    ctx.sync_status()


@pytest.mark.parametrize("dim", [64, 90])
def test_norm_position_outside_the_table(ctx, dim):
    import torch
    from paper_2505_23725_b200 import binding
    q, k, cos, sin, pos, gq, gk, _, _ = _qk_inputs((40, 4, 2, dim, dim, False), torch.float32)
    want, _ = ctx.qk_norm_rope(q, k, cos, sin, pos, gq, gk)
    for bad in (-1, cos.shape[0], 1 << 40):
        p = pos.clone()
        p[17] = bad
        got, _ = ctx.qk_norm_rope(q, k, cos, sin, p, gq, gk)
        with pytest.raises(binding.MulocoError) as e:
            ctx.sync_status()
        assert e.value.status == binding.EINVAL and "position" in str(e.value)
        assert torch.isnan(got[17]).all()
        rest = [i for i in range(40) if i != 17]
        assert torch.equal(got[rest], want[rest])
    ctx.sync_status()


def test_norm_refusals(ctx):
    import torch
    from paper_2505_23725_b200 import binding
    q, k, cos, sin, pos, gq, gk, dqo, dko = _qk_inputs((8, 4, 2, 64, 64, False), torch.float32)
    for bad in (dict(q=q.half()), dict(q=q[..., ::2]), dict(k=k[:5]), dict(cos=cos[:, :4]), dict(gain_q=gq[:10]),
                dict(positions=pos.int()), dict(q=q.cpu()), dict(k=k.bfloat16()), dict(q=None, k=None),
                dict(q=q.view(8, -1))):
        args = {**dict(q=q, k=k, cos=cos, sin=sin, positions=pos, gain_q=gq, gain_k=gk), **bad}
        with pytest.raises(ValueError):
            ctx.qk_norm_rope(**args)
    with pytest.raises(ValueError):
        ctx.qk_norm_rope_backward(dqo[:4], dko, q, k, cos, sin)
    with pytest.raises(binding.MulocoError) as e:              # odd head size
        ctx.qk_norm_rope(q[..., :63], None, cos, sin)
    assert e.value.status == binding.ESHAPE
    with pytest.raises(binding.MulocoError) as e:              # rotated part larger than the head
        ctx.qk_norm_rope(q[..., :32], None, cos, sin)
    assert e.value.status == binding.ESHAPE
    with pytest.raises(binding.MulocoError) as e:              # more tokens than table rows, no positions
        ctx.qk_norm_rope(q, k, cos[:4].contiguous(), sin[:4].contiguous())
    assert e.value.status == binding.ESHAPE
    with pytest.raises(binding.MulocoError) as e:
        ctx.qk_norm_rope(q, k, cos, sin, eps=-1.0)
    assert e.value.status == binding.EINVAL


# ------------------------------------------------------------------------------------------------
# gated feed-forward block
# ------------------------------------------------------------------------------------------------
FFN_SHAPES = [(1, 8, 8), (1, 64, 128), (7, 768, 2048), (16, 72, 200), (17, 128, 352), (33, 136, 1000), (64, 264, 136),
              (65, 128, 264), (128, 200, 520), (129, 200, 520), (200, 1024, 392), (256, 328, 1384), (257, 328, 1384),
              (513, 128, 704), (1030, 264, 520)]


def _ffn_inputs(T, d, F, seed=0):
    rng = np.random.default_rng(seed + T + d + F)
    return (_bf16(rng, T, d), _bf16(rng, d, F, scale=d ** -0.5), _bf16(rng, d, F, scale=d ** -0.5),
            _bf16(rng, F, d, scale=F ** -0.5), _bf16(rng, T, d))


def _check_ffn(ctx, x, w1, w3, w2, dy, act):
    y, (g, u, h) = ctx.gated_ffn(x, w1, w3, w2, activation=act)
    grads = ctx.gated_ffn_backward(dy, x, w1, w3, w2, (g, u, h), activation=act)
    ctx.sync_status()
    X, W1, W3, W2, DY = (_np(t) for t in (x, w1, w3, w2, dy))
    (T, d), F = X.shape, W1.shape[1]
    _, G, U, H = O.gated_ffn(X, W1, W3, W2, act)
    dG, dU = d * 2.0 ** -23 * (np.abs(X) @ np.abs(W1)), d * 2.0 ** -23 * (np.abs(X) @ np.abs(W3))
    _within(g, G, dG + U16 * np.abs(G), "g")
    _within(u, U, dU + U16 * np.abs(U), "u")
    value, slope = O.activation(G, act)
    # the slope of either activation is below 1.13; a few units in the last place for the activation itself
    dH = 1.2 * dG * np.abs(U) + dU * np.abs(value) + 1.2 * dG * dU + 16 * U32 * np.abs(G * U)
    _within(h, H, dH + U16 * (np.abs(H) + dH), "h")
    # the later products start from the library's own rounded tensors
    Gr, Ur, Hr = _np(g), _np(u), _np(h)
    Y = Hr @ W2
    _within(y, Y, F * 2.0 ** -23 * (np.abs(Hr) @ np.abs(W2)) + U16 * np.abs(Y) * 1.01, "y")
    DX, DW1, DW3, DW2, DGr, DUr = O.gated_ffn_backward(DY, X, W1, W3, W2, Gr, Ur, Hr, act)
    value, slope = O.activation(Gr, act)
    dDH = d * 2.0 ** -23 * (np.abs(DY) @ np.abs(W2.T))
    # what dG and dU are off by before they are multiplied: their sum, the activation's few units (of at most |g| sigma (1 - sigma) + 1
    # for the slope) and their rounding
    eG = dDH * np.abs(Ur * slope) + 32 * U32 * np.abs((DY @ W2.T) * Ur) * (1 + np.abs(Gr)) + U16 * np.abs(DGr) * 1.01
    eU = dDH * np.abs(value) + 32 * U32 * np.abs((DY @ W2.T) * Gr) + U16 * np.abs(DUr) * 1.01
    aG, aU = np.abs(DGr) + eG, np.abs(DUr) + eU
    bounds = (eG @ np.abs(W1.T) + eU @ np.abs(W3.T) + 2 * F * 2.0 ** -23 * (aG @ np.abs(W1.T) + aU @ np.abs(W3.T)),
              np.abs(X.T) @ (eG + T * 2.0 ** -23 * aG), np.abs(X.T) @ (eU + T * 2.0 ** -23 * aU),
              T * 2.0 ** -23 * (np.abs(Hr.T) @ np.abs(DY)))
    for name, got, ref, b in zip(("dx", "dw1", "dw3", "dw2"), grads, (DX, DW1, DW3, DW2), bounds):
        _within(got, ref, b + U16 * (np.abs(ref) + b), name)
        # the entrywise bounds add magnitudes; in norm the two independent roundings give about 2.4e-3
        rel = np.linalg.norm(_np(got) - ref) / max(np.linalg.norm(ref), 1e-30)
        assert rel < 4e-3, f"{name}: {rel:.2e}"
    return y, (g, u, h), grads


@pytest.mark.parametrize("shape", FFN_SHAPES, ids=str)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn(ctx, shape, act):
    x, w1, w3, w2, dy = _ffn_inputs(*shape)
    _check_ffn(ctx, x, w1, w3, w2, dy, act)


def test_gated_ffn_without_saving_and_repeatable(ctx):
    import torch
    for T in (5, 128, 700):
        x, w1, w3, w2, dy = _ffn_inputs(T, 264, 520)
        y, saved = ctx.gated_ffn(x, w1, w3, w2)
        y2, none = ctx.gated_ffn(x, w1, w3, w2, save=False)
        assert none is None and torch.equal(y, y2)
        a = ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved)
        b = ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    ctx.sync_status()


@pytest.mark.parametrize("T", [3, 200])
def test_gated_ffn_strided(ctx, T):
    """Activations and weights as parts of wider matrices."""
    import torch
    x, w1, w3, w2, dy = _ffn_inputs(T, 136, 264)
    wide = torch.zeros(T, 136 + 24, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:144] = x
    both = torch.cat([w1, w3], 1)
    tall = torch.zeros(264, 200, dtype=torch.bfloat16, device="cuda")
    tall[:, 16:152] = w2
    dwide = torch.zeros(T, 152, dtype=torch.bfloat16, device="cuda")
    dwide[:, 16:] = dy
    got = _check_ffn(ctx, wide[:, 8:144], both[:, :264], both[:, 264:], tall[:, 16:152], dwide[:, 16:], "silu")
    want = _check_ffn(ctx, x, w1, w3, w2, dy, "silu")
    assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(got[2], want[2]))


def test_gated_ffn_of_no_tokens(ctx):
    x, w1, w3, w2, dy = _ffn_inputs(0, 64, 128)
    y, saved = ctx.gated_ffn(x, w1, w3, w2)
    dx, dw1, dw3, dw2 = ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved)
    ctx.sync_status()
    assert y.shape == (0, 64) and dx.shape == (0, 64)
    assert not dw1.any() and not dw3.any() and not dw2.any()   # empty sums


@pytest.mark.parametrize("T", [9, 300])
def test_gated_ffn_extreme_values(ctx, T):
    """Gates far to either side: act -> 0 or g, and no NaN; a NaN token stays in its row."""
    import torch
    x, w1, w3, w2, dy = _ffn_inputs(T, 64, 128)
    x[2] *= 200
    _, (g, u, h) = ctx.gated_ffn(x, w1, w3, w2)
    assert g.abs().max() > 100 and torch.isfinite(h.float()).all()
    x[4] = float("nan")
    y, (g, u, h) = ctx.gated_ffn(x, w1, w3, w2)
    assert torch.isnan(y[4]).all()
    rest = [i for i in range(T) if i != 4]
    assert torch.isfinite(y[rest].float()).all()
    ctx.sync_status()


def test_gated_ffn_refusals(ctx):
    import torch
    from paper_2505_23725_b200 import binding
    x, w1, w3, w2, dy = _ffn_inputs(4, 64, 128)
    saved = ctx.gated_ffn(x, w1, w3, w2)[1]
    for bad in (dict(x=x.float()), dict(x=x[:, :56]), dict(w3=w3[:, :64]), dict(w2=w2.t()), dict(w1=w1.cpu()),
                dict(activation="relu")):
        with pytest.raises(ValueError):
            ctx.gated_ffn(**{**dict(x=x, w1=w1, w3=w3, w2=w2), **bad})
    with pytest.raises(ValueError):
        ctx.gated_ffn_backward(dy[:2], x, w1, w3, w2, saved)
    with pytest.raises(ValueError):
        ctx.gated_ffn_backward(dy, x, w1, w3, w2, tuple(t[:2] for t in saved))
    with pytest.raises(binding.MulocoError) as e:              # widths that are not multiples of 8
        ctx.gated_ffn(x[:, :60].contiguous(), w1[:60], w3[:60], w2[:, :60].contiguous())
    assert e.value.status == binding.ESHAPE
    with pytest.raises(binding.MulocoError) as e:              # rows that do not start on 16 bytes
        ctx.gated_ffn(torch.zeros(4, 68, dtype=torch.bfloat16, device="cuda")[:, :64], w1, w3, w2)
    assert e.value.status == binding.ESHAPE
    with pytest.raises(binding.MulocoError) as e:
        ctx.gated_ffn(torch.zeros(4, 72, dtype=torch.bfloat16, device="cuda")[:, 4:68], w1, w3, w2)
    assert e.value.status == binding.EINVAL


# ------------------------------------------------------------------------------------------------
# the two ways of a call
# ------------------------------------------------------------------------------------------------
def test_compiled_and_python_call_paths_agree(ctx):
    """A call marshalled by the compiled module and one marshalled in Python give the same tensors; the suite runs with
    the compiled one (it has to be there), and what it does not take goes the other way."""
    import torch
    from paper_2505_23725_b200 import binding
    plain = binding.Context("cuda:0")
    plain._fast = {}
    assert set(ctx._fast) == {"qk_norm_rope", "qk_norm_rope_backward", "gated_ffn", "gated_ffn_backward", "adamw_step",
                              "adamw_moments"}
    outs = []
    for owner in (ctx, plain):
        torch.manual_seed(3)
        p, g = torch.randn(5000, device="cuda"), torch.randn(5000, device="cuda")
        opt = binding.AdamW(owner, [p], grads=[g], state_bits=8, **HYPER)
        opt.step()
        opt.step(lr_scale=0.5)
        outs.append((p, *opt.moments(), opt.state1))
        assert opt.steps == 2
        opt.close()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    q, k, cos, sin, pos, gq, gk, dqo, dko = _qk_inputs((37, 6, 2, 64, 32, False), torch.bfloat16, layout="wide")
    for args in ((q, k, cos, sin, pos, gq, gk, 1e-5, True), (q, None, cos, sin), (None, k, cos, sin, pos, None, gk)):
        assert ctx._quick("qk_norm_rope", *(args + (None,) * (7 - len(args)) + (1e-6, False) if len(args) < 9 else args)) is not None
        for a, b in zip(ctx.qk_norm_rope(*args), plain.qk_norm_rope(*args)):
            assert (a is None and b is None) or (torch.equal(a, b) and a.stride() == b.stride())
        dy = (dqo if args[0] is not None else None, dko if args[1] is not None else None)
        for a, b in zip(ctx.qk_norm_rope_backward(*dy, *args), plain.qk_norm_rope_backward(*dy, *args)):
            assert (a is None and b is None) or torch.equal(a, b)
    x, w1, w3, w2, dy = _ffn_inputs(21, 72, 136)
    y, saved = ctx.gated_ffn(x, w1, w3, w2, "gelu")
    y2, saved2 = plain.gated_ffn(x, w1, w3, w2, "gelu")
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(saved, saved2))
    for a, b in zip(ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved, "gelu"), plain.gated_ffn_backward(dy, x, w1, w3, w2, saved, "gelu")):
        assert torch.equal(a, b)
    assert ctx._quick("gated_ffn", x.float(), w1, w3, w2, 0, True) is None
    with torch.cuda.stream(torch.cuda.Stream()):
        assert ctx._quick("gated_ffn", x, w1, w3, w2, 0, True) is None
    ctx.sync_status()
    plain.sync_status()
    plain.close()


# ------------------------------------------------------------------------------------------------
# streams
# ------------------------------------------------------------------------------------------------
def test_operators_from_another_stream():
    """Inputs made and results used on a stream that is not the context's."""
    import torch
    from paper_2505_23725_b200 import binding
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = binding.Context("cuda:0", stream=own)
    want = binding.Context("cuda:0")
    with torch.cuda.stream(other):
        for i in range(5):
            torch.manual_seed(i)
            big = torch.randn(2048, 2048, device="cuda")
            x = (big @ big)[:512, :256].to(torch.bfloat16).contiguous() / 64      # still running when the call is made
            w1, w3 = (torch.randn(256, 512, device="cuda").to(torch.bfloat16) / 16 for _ in range(2))
            w2 = torch.randn(512, 256, device="cuda").to(torch.bfloat16) / 16
            y, saved = ctx.gated_ffn(x, w1, w3, w2)
            total = y.float().sum()
            q = x.view(512, 4, 64)
            cos, sin = torch.ones(512, 32, device="cuda"), torch.zeros(512, 32, device="cuda")
            n, _ = ctx.qk_norm_rope(q, None, cos, sin)
            nsum = n.float().sum()
            p = torch.ones(4096, device="cuda")
            opt = binding.AdamW(ctx, [p], grads=[big.view(-1)[:4096]], state_bits=8)
            opt.step()
            psum = p.sum()
            other.synchronize()
            y0, _ = want.gated_ffn(x, w1, w3, w2)      # `want` lives on the default stream
            n0, _ = want.qk_norm_rope(q, None, cos, sin)
            torch.cuda.synchronize()
            assert torch.equal(y, y0) and torch.equal(n, n0)
            assert total.item() == y0.float().sum().item() and nsum.item() == n0.float().sum().item()
            assert psum.item() == p.sum().item() and not torch.equal(p, torch.ones_like(p))
            opt.close()
    ctx.sync_status()
    ctx.close()
    want.close()
