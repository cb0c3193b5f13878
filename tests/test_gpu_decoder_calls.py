"""Attention, layer norm and embedding on a B200 as calls: what they refuse, values that are not finite, streams, captured graphs,
call paths, waits that run out, and a decoder block made of them."""
import ctypes as C

import pytest
import torch

from paper_2505_23725_b200 import binding, layers

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.close()


def rand(*shape, dtype=BF16, seed=None, s=1.0):
    g = None if seed is None else torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, device="cuda", generator=g) * s).to(dtype)


def qkv(T, hq=4, hk=2, D=64, seed=0):
    return rand(T, hq, D, seed=seed), rand(T, hk, D, seed=seed + 1), rand(T, hk, D, seed=seed + 2), rand(T, hq, D, seed=seed + 3)


def everything(c, seq, q, k, v, do, x, r, w, b, ids, table):
    o, lse = c.causal_attention(q, k, v, seq)
    y, h, rstd, mean = c.layer_norm(x, w, b, r)
    return [o, lse, *c.causal_attention_backward(do, q, k, v, o, lse, seq), y, h, rstd, mean,
            *c.layer_norm_backward(x, h, rstd, mean, w, r, True), c.embedding(ids, table, 0.5),
            c.embedding_backward(x, ids, table.shape[0], 0.5, torch.float32),
            c.embedding_backward(x, ids, table.shape[0], 0.5, BF16)]


def inputs(T=333, d=200, V=50, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    return [*qkv(T, seed=seed), rand(T, d, seed=seed + 4), rand(T, d, seed=seed + 5), rand(d, dtype=torch.float32, seed=seed + 6),
            rand(d, dtype=torch.float32, seed=seed + 7), ids, rand(V, d, seed=seed + 8)]


LENGTHS = [100, 0, 140, 70]                  # of 333 tokens


def test_refusals(ctx):
    q, k, v, do = qkv(40)
    seq = binding.Sequences(ctx, [40])
    o, lse = ctx.causal_attention(q, k, v, seq)

    def status(call, code):
        with pytest.raises(binding.MulocoError) as e:
            call()
        assert e.value.status == code, str(e.value)

    for bad in ([41], [20, 30], [-1, 5]):
        status(lambda: binding.Sequences(ctx, bad, tokens=40), binding.ESHAPE)
    for heads in ((4, 3), (2, 4)):
        a, b, c, _ = qkv(40, *heads)
        status(lambda: ctx.causal_attention(a, b, c, seq), binding.ESHAPE)
    for D in (4, 12, 136, 256):
        a, b, c, _ = qkv(40, D=D)
        status(lambda: ctx.causal_attention(a, b, c, seq), binding.ESHAPE)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        status(lambda: ctx.causal_attention(q, k, v, seq, scale=scale), binding.EINVAL)
    status(lambda: ctx.causal_attention(q, k[:, :1].expand(40, 2, 64), v, seq), binding.ESHAPE)       # heads that overlap
    status(lambda: ctx.causal_attention(rand(40, 4, 68)[:, :, :64], k, v, seq), binding.ESHAPE)       # strides that are no multiple of 8
    status(lambda: ctx.causal_attention(rand(40, 4, 72)[:, :, 4:68], k, v, seq), binding.EINVAL)      # not on 16 bytes
    status(lambda: ctx.causal_attention_backward(rand(40, 4, 68)[:, :, :64], q, k, v, o, lse, seq), binding.ESHAPE)
    for args in ((q.float(), k, v), (q, k[:39], v), (q, k, v[:, :, :56]), (q[:39], k[:39], v[:39]), (q.cpu(), k, v), (q[0], k, v)):
        with pytest.raises((ValueError, IndexError)):
            ctx.causal_attention(*args, seq)
    with pytest.raises(ValueError):
        ctx.causal_attention_backward(do, q, k, v, o.transpose(0, 1), lse, seq)
    with pytest.raises(ValueError):
        ctx.causal_attention_backward(do, q, k, v, o, lse.double(), seq)
    other = binding.Context("cuda:0")
    with pytest.raises(ValueError, match="another context"):
        other.causal_attention(q, k, v, seq)
    theirs = binding.Sequences(other, [40])
    other.close()
    with pytest.raises(RuntimeError, match="closed"):
        other.layer_norm(rand(3, 8))
    with pytest.raises(RuntimeError, match="closed"):
        ctx.causal_attention(q, k, v, theirs)
    with pytest.raises(RuntimeError, match="closed"):
        binding.Sequences(other, [3])

    x = rand(5, 16)
    w = torch.ones(16, device="cuda")
    for args in ((x.half(),), (x[0],), (x, w[:15]), (x, w.to(BF16)), (x, None, w[::2]), (x, None, None, x.float()), (x.t(),), (x.cpu(),)):
        with pytest.raises(ValueError):
            ctx.layer_norm(*args)
    status(lambda: ctx.layer_norm(x, eps=-1.0), binding.EINVAL)
    status(lambda: ctx.layer_norm(rand(2, 32769)), binding.ESHAPE)
    status(lambda: ctx.layer_norm(x[:1].expand(5, 16)), binding.ESHAPE)
    y, h, rstd, mean = ctx.layer_norm(x)
    for args in ((x.float(), h, rstd, mean), (x, h, rstd[:4], mean), (x, h, rstd, mean.double()), (x[:4], h, rstd, mean)):
        with pytest.raises(ValueError):
            ctx.layer_norm_backward(*args)

    ids, table = torch.zeros(6, dtype=torch.int64, device="cuda"), rand(9, 16)
    for args in ((ids.int(), table), (ids[None], table), (ids, table.half()), (ids, table.t()), (ids.cpu(), table), (ids.repeat(2)[::2], table)):
        with pytest.raises(ValueError):
            ctx.embedding(*args)
    for args in ((rand(5, 16), ids, 9), (rand(6, 16).half(), ids, 9), (rand(6, 16), ids.int(), 9)):
        with pytest.raises(ValueError):
            ctx.embedding_backward(*args)
    with pytest.raises(ValueError):
        ctx.embedding_backward(rand(6, 16), ids, 9, dtype=torch.float16)
    status(lambda: ctx.embedding(ids, table, scale=float("inf")), binding.EINVAL)
    ctx.sync_status()
    assert torch.equal(ctx.causal_attention(q, k, v, seq)[0], o)


def test_refusals_of_the_library(ctx):
    """What the binding itself does not let through: pointers and sizes of a C caller."""
    lib, size, handle = ctx.lib, C.c_size_t(), C.c_void_p()
    lengths = (C.c_int64 * 2)(3, 4)
    assert lib.muloco_sequences_bytes(ctx.ctx, lengths, 2, 7, None) == binding.EINVAL
    assert lib.muloco_sequences_bytes(ctx.ctx, None, 2, 7, C.byref(size)) == binding.EINVAL
    assert lib.muloco_sequences_bytes(ctx.ctx, lengths, 2, 2 ** 31, C.byref(size)) == binding.ESHAPE
    assert lib.muloco_sequences_bytes(ctx.ctx, lengths, 2, 7, C.byref(size)) == binding.OK and size.value == 2 * 3 * 16
    table = torch.empty(size.value + 16, dtype=torch.uint8, device="cuda")
    for p, n in ((None, size.value), (table.data_ptr() + 8, size.value), (table.data_ptr(), size.value - 1)):
        assert lib.muloco_sequences_create(ctx.ctx, lengths, 2, 7, p, n, C.byref(handle)) == binding.EINVAL and not handle
    assert lib.muloco_sequences_create(ctx.ctx, lengths, 2, 7, table.data_ptr(), size.value, None) == binding.EINVAL
    seq = binding.Sequences(ctx, [3, 4])
    q, k, v, do = qkv(7)
    a = ctx._attention(q, k, v, seq, 0.1)
    o, lse = torch.empty_like(q), torch.empty(4, 7, device="cuda")
    assert lib.muloco_causal_attention(ctx.ctx, a, None, o.data_ptr(), lse.data_ptr()) == binding.EINVAL
    assert lib.muloco_causal_attention(ctx.ctx, a, seq.handle, None, lse.data_ptr()) == binding.EINVAL
    assert lib.muloco_causal_attention(ctx.ctx, a, seq.handle, o.data_ptr() + 2, lse.data_ptr()) == binding.EINVAL
    some = [o.data_ptr(), lse.data_ptr(), lse.data_ptr(), o.data_ptr(), k.data_ptr(), v.data_ptr()]
    for i in range(6):
        args = [None if j == i else p for j, p in enumerate(some)]
        assert lib.muloco_causal_attention_backward(ctx.ctx, a, seq.handle, do.data_ptr(), *do.stride()[:2], *args) == binding.EINVAL
    x = rand(3, 8)
    n = ctx._norm(x, None, None, x, "residual", 1e-6, True)
    f = torch.empty(8, device="cuda")
    assert lib.muloco_layer_norm(ctx.ctx, n, None, x.data_ptr(), f.data_ptr(), f.data_ptr()) == binding.EINVAL          # no h
    assert lib.muloco_layer_norm(ctx.ctx, n, o.data_ptr(), o.data_ptr(), f.data_ptr(), f.data_ptr()) == binding.EINVAL  # y is h
    assert lib.muloco_layer_norm_backward(ctx.ctx, n, x.data_ptr(), 8, f.data_ptr(), f.data_ptr(), o.data_ptr(), f.data_ptr(), None,
                                          None) == binding.EINVAL                                                        # no scratch
    e = binding._EMBEDDING_PACK(3, 4, 8, 8, binding.BF16, 1.0, 0)
    assert lib.muloco_embedding_lookup(ctx.ctx, e, x.data_ptr(), o.data_ptr()) == binding.EINVAL
    assert lib.muloco_embedding_scratch(ctx.ctx, -1, 8, C.byref(size)) == binding.EINVAL
    ctx.sync_status()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_other_sequences_and_padding_may_hold_anything(ctx, bad):
    """Sequences that end inside a tile, their neighbours and the tokens behind the last one not finite."""
    lengths, T = [70, 129, 130, 200], 560
    q, k, v, do = qkv(T, D=128, seed=5)
    seq = binding.Sequences(ctx, lengths, tokens=T)
    o, lse = ctx.causal_attention(q, k, v, seq)
    want = [o, lse.t(), *ctx.causal_attention_backward(do, q, k, v, o, lse, seq)]
    spoilt = [t.clone() for t in (q, k, v, do)]
    for t in spoilt:
        t[70:199] = bad
        t[529:] = bad
    o2, lse2 = ctx.causal_attention(*spoilt[:3], seq)
    o3, lse3 = o.clone(), lse.clone()
    o3[70:199], o3[529:], lse3[:, 70:199], lse3[:, 529:] = bad, bad, bad, bad
    got = [o2, lse2.t(), *ctx.causal_attention_backward(spoilt[3], *spoilt[:3], o3, lse3, seq)]
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[70:199] = False
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(o2[70:199].float()).any()
    ctx.sync_status()


def test_a_key_that_is_not_finite_spoils_the_queries_behind_it(ctx):
    q, k, v, do = qkv(300, 2, 2, 64, seed=9)
    seq = binding.Sequences(ctx, [300])
    want, _ = ctx.causal_attention(q, k, v, seq)
    for bad in (float("nan"), float("inf")):
        k2 = k.clone()
        k2[140, 1, 3] = bad
        o, lse = ctx.causal_attention(q, k2, v, seq)
        assert torch.equal(o[:, 0], want[:, 0]) and torch.equal(o[:140, 1], want[:140, 1])
        if bad != bad:
            assert torch.isnan(o[140:, 1].float()).all() and torch.isnan(lse[1, 140:]).all()


def test_rows_that_are_not_finite(ctx):
    """A norm's row is its own; a token's gradient reaches its row of the table only."""
    x = rand(200, 96, seed=1)
    y, _, _, _ = ctx.layer_norm(x)
    x2 = x.clone()
    x2[7, 3], x2[150, 0] = float("nan"), float("inf")
    y2, h, rstd, mean = ctx.layer_norm(x2)
    keep = torch.ones(200, dtype=torch.bool, device="cuda")
    keep[[7, 150]] = False
    assert torch.equal(y2[keep], y[keep]) and torch.isnan(y2[7].float()).all()
    ids = torch.arange(200, device="cuda") % 11
    g, g2 = ctx.embedding_backward(x, ids, 11), ctx.embedding_backward(x2, ids, 11)
    rows = torch.arange(11, device="cuda")
    good = (rows != 7) & (rows != 150 % 11)
    assert torch.equal(g[good], g2[good]) and torch.isnan(g2[7, 3]) and torch.isinf(g2[150 % 11, 0])


def test_compiled_and_python_call_paths_agree(ctx):
    plain = binding.Context("cuda:0")
    plain._fast, plain._fast_decoder = {}, {}
    assert set(ctx._fast_decoder) == {"causal_attention", "causal_attention_backward", "layer_norm", "layer_norm_backward",
                                      "embedding_lookup", "embedding_backward"}
    args = inputs()
    for a, b in zip(everything(ctx, binding.Sequences(ctx, LENGTHS, 333), *args),
                    everything(plain, binding.Sequences(plain, LENGTHS, 333), *args)):
        assert torch.equal(a, b) and a.stride() == b.stride() and a.dtype == b.dtype
    plain.sync_status()
    plain.close()


def test_results_do_not_change_from_run_to_run(ctx):
    args = inputs(seed=3)
    seq = binding.Sequences(ctx, LENGTHS, 333)
    want = everything(ctx, seq, *args)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(everything(ctx, seq, *args), want))


def test_on_another_stream_than_the_context(ctx):
    args = inputs(seed=4)
    want = everything(ctx, binding.Sequences(ctx, LENGTHS, 333), *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            torch.cuda._sleep(2_000_000)     # what is made here is late
            late = [t.clone() for t in args]
            got = everything(ctx, binding.Sequences(ctx, LENGTHS, 333), *late)
            copies = [t.clone() for t in got]
            del late, got
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want))
    ctx.sync_status()


def test_inside_captured_graphs(ctx):
    """Two graphs of one context, replayed in turn on other values; sequences are made outside."""
    args = inputs(seed=6)
    side = torch.cuda.Stream()
    mine = binding.Context("cuda:0", stream=side)
    seq = binding.Sequences(mine, LENGTHS, 333)
    with torch.cuda.stream(side):
        everything(mine, seq, *args)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = everything(mine, seq, *args)
            with pytest.raises(binding.MulocoError) as e:
                binding.Sequences(mine, LENGTHS, 333)
            assert e.value.status == binding.ESTATE
        graphs.append((graph, out))
    here = binding.Sequences(ctx, LENGTHS, 333)
    for seed in (7, 8):
        for t, new in zip(args, inputs(seed=seed)):
            t.copy_(new)
        want = everything(ctx, here, *args)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
    mine.sync_status()
    del graphs, graph, out
    mine.close()


def test_waits_run_out():
    """A copy left out on purpose: the call ends, the status says so, and the context goes on."""
    mine = binding.Context("cuda:0")
    q, k, v, do = qkv(700, 2, 2, 64)
    seq = binding.Sequences(mine, [700])
    o, lse = mine.causal_attention(q, k, v, seq)
    want = mine.causal_attention_backward(do, q, k, v, o, lse, seq)
    mine.sync_status()
    for call in (lambda: mine.causal_attention(q, k, v, seq), lambda: mine.causal_attention_backward(do, q, k, v, o, lse, seq)):
        mine._check(mine.lib.muloco_debug_set(mine.ctx, binding.DEBUG_WAIT_LIMIT_NS, 2_000_000))
        mine._check(mine.lib.muloco_debug_set(mine.ctx, binding.DEBUG_WITHHOLD_COPY, 1))
        call()
        with pytest.raises(binding.MulocoError) as e:
            mine.sync_status()
        assert e.value.status == binding.ETIMEOUT
        mine._check(mine.lib.muloco_debug_set(mine.ctx, binding.DEBUG_WAIT_LIMIT_NS, 0))
        assert torch.equal(mine.causal_attention(q, k, v, seq)[0], o)
        assert all(torch.equal(a, b) for a, b in zip(mine.causal_attention_backward(do, q, k, v, o, lse, seq), want))
        mine.sync_status()
    mine.close()


def test_calls_allocate_nothing_of_their_own(ctx):
    args = inputs(seed=2)
    seq = binding.Sequences(ctx, LENGTHS, 333)
    for _ in range(2):
        out = everything(ctx, seq, *args)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    del out
    everything(ctx, seq, *args)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


def test_many_sequences_of_one_token(ctx):
    """More units than the grid has places for, each a row of its own: o is v, nothing flows into q and k."""
    T = 3000
    q, k, v, do = qkv(T, 4, 2, 64, seed=11)
    lengths = [1, 0] * T
    seq = binding.Sequences(ctx, lengths)
    o, lse = ctx.causal_attention(q, k, v, seq)
    assert torch.equal(o, v.repeat_interleave(2, 1))
    dq, dk, dv = ctx.causal_attention_backward(do, q, k, v, o, lse, seq)
    # ds = p (dp - p dp), p within 2^-18 of 1 (the scores' rounding): 2^-18 of the products' magnitudes
    dp = (do.float().abs() * v.float().abs().repeat_interleave(2, 1)).sum(2, keepdim=True)
    assert (dq.float().abs() <= 2.0 ** -18 * dp * k.float().abs().repeat_interleave(2, 1) + 1e-30).all()
    want = do.double().view(T, 2, 2, 64).sum(2)
    size = do.double().abs().view(T, 2, 2, 64).sum(2)
    assert ((dv.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -16) * size).all()
    ctx.sync_status()


def test_results_in_place_of_inputs(ctx):
    """What the header allows a C caller: y or h over x, or over the residual."""
    x, r = rand(300, 1000, seed=1), rand(300, 1000, seed=2)
    want, h, rstd, mean = ctx.layer_norm(x, residual=r)
    for y_over, h_over in (("x", "r"), ("r", "x"), (None, "x"), ("x", None)):
        t = dict(x=x.clone(), r=r.clone())
        y, hh = (t[o] if o else torch.empty_like(x) for o in (y_over, h_over))
        a = ctx._norm(t["x"], None, None, t["r"], "residual", 1e-6, True)
        assert ctx.lib.muloco_layer_norm(ctx.ctx, a, hh.data_ptr(), y.data_ptr(), torch.empty_like(mean).data_ptr(),
                                         torch.empty_like(rstd).data_ptr()) == binding.OK
        assert torch.equal(y, want) and torch.equal(hh, h)
    wide = rand(300, 1008)
    a = ctx._norm(wide[:, :1000], None, None, None, "residual", 1e-6, False)
    assert ctx.lib.muloco_layer_norm(ctx.ctx, a, None, wide.data_ptr(), None, rstd.data_ptr()) == binding.EINVAL


def test_offsets_beyond_32_bits(ctx):
    """Tensors of more than 2^31 entries: their last rows come out as on their own."""
    heads, dim, last = 120, 128, 200
    lengths = [128] * 1100 + [last]
    T = sum(lengths)
    assert T * heads * dim > 2 ** 31
    q, k, v, do = (torch.zeros(T, heads, dim, dtype=BF16, device="cuda") for _ in range(4))
    for i, t in enumerate((q, k, v, do)):
        t[-last:] = rand(last, heads, dim, seed=i)
    seq, own = binding.Sequences(ctx, lengths), binding.Sequences(ctx, [last])
    o, lse = ctx.causal_attention(q, k, v, seq)
    tails = [t[-last:].clone() for t in (q, k, v, do)]
    o2, lse2 = ctx.causal_attention(*tails[:3], own)
    assert torch.equal(o[-last:], o2) and torch.equal(lse[:, -last:], lse2)
    got = ctx.causal_attention_backward(do, q, k, v, o, lse, seq)
    for a, b in zip(got, ctx.causal_attention_backward(tails[3], *tails[:3], o2, lse2, own)):
        assert torch.equal(a[-last:], b) and not a[:100].any()
    del q, k, v, do, o, got
    d = 2048
    rows = 2 ** 31 // d + 300
    x = torch.zeros(rows, d, dtype=BF16, device="cuda")
    x[-50:] = rand(50, d, seed=5)
    y, _, rstd, mean = ctx.layer_norm(x)
    assert torch.equal(y[-50:], ctx.layer_norm(x[-50:].clone())[0])
    w = torch.ones(d, device="cuda")
    dx, _, _ = ctx.layer_norm_backward(x, x, rstd, mean, weight=w)
    assert torch.equal(dx[-50:], ctx.layer_norm_backward(*(t[-50:].clone() for t in (x, x, rstd, mean)), weight=w)[0])
    del y, dx
    ids = torch.tensor([rows - 1, 3, rows - 30, rows - 1], device="cuda")
    assert torch.equal(ctx.embedding(ids, x), x[ids])
    g = rand(4, d, seed=6)
    grad = ctx.embedding_backward(g, ids, rows, dtype=BF16)
    assert torch.equal(grad[rows - 30], g[2]) and torch.equal(grad[rows - 1], (g[0].float() + g[3].float()).to(BF16))
    assert not grad[rows - 29:rows - 1].any()
    ctx.sync_status()


def test_two_graphs_side_by_side():
    """Graphs of two contexts replayed on two streams at once: no workspace is shared."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    owners = [binding.Context("cuda:0", stream=s) for s in streams]
    sets = [inputs(seed=20 + i) for i in range(2)]
    seqs = [binding.Sequences(o, LENGTHS, 333) for o in owners]
    torch.cuda.synchronize()
    graphs, outs, wants = [], [], []
    for s, o, q, a in zip(streams, owners, seqs, sets):
        with torch.cuda.stream(s):
            wants.append([t.clone() for t in everything(o, q, *a)])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(everything(o, q, *a))
        graphs.append(g)
    for _ in range(30):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for out, want in zip(outs, wants):
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    for o in owners:
        o.sync_status()
    del graphs, g, outs, out
    for o in owners:
        o.close()


def block(ops, p, ids, seq, cos, sin, heads):
    """A decoder block as they are used together: embedding, norm, rotation, attention, norm with the stream, feed-forward."""
    T, dim = ids.shape[0], cos.shape[1] * 2
    stream = ops.embedding(ids, p["embed"], 2.0)
    n = ops.norm(stream, p["g1"])
    q, k, v = ((n @ p[w]).view(T, h, dim) for w, h in zip(("wq", "wk", "wv"), heads))
    q, k = ops.rope(q, k, cos, sin, seq)
    a = ops.attention(q, k, v, seq).reshape(T, -1)
    n, stream = ops.norm(a @ p["wo"], p["g2"], stream)
    y = ops.ffn(n, p["w1"], p["w3"], p["w2"])
    return ops.norm(y, p["g3"], stream)[0]


class Library:
    def __init__(self, owner):
        self.o = owner

    def embedding(self, ids, t, s):
        return layers.embedding(self.o, ids, t, s)

    def norm(self, x, g, stream=None):
        return layers.layer_norm(self.o, x, g, residual=stream, center=False)

    def rope(self, q, k, cos, sin, seq):
        return layers.qk_norm_rope(self.o, q, k, cos, sin, seq.positions)

    def attention(self, q, k, v, seq):
        return layers.causal_attention(self.o, q, k, v, seq)

    def ffn(self, *a):
        return layers.gated_ffn(self.o, *a)


class Definition:
    """The same in 64 bits."""

    def embedding(self, ids, t, s):
        return t[ids] * s

    def norm(self, x, g, stream=None):
        h = x if stream is None else x + stream
        y = h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * g
        return y if stream is None else (y, h)

    def rope(self, q, k, cos, sin, seq):
        c, s = cos.double()[seq.positions][:, None], sin.double()[seq.positions][:, None]

        def turned(x):
            x = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            a, b = x.chunk(2, -1)
            return torch.cat((a * c - b * s, b * c + a * s), -1)
        return turned(q), turned(k)

    def attention(self, q, k, v, seq):
        out, at = [], 0
        group = q.shape[1] // k.shape[1]
        for n in seq.lengths:
            a, b, c = (t[at:at + n].transpose(0, 1) for t in (q, k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)))
            s = (a @ b.transpose(1, 2) * q.shape[2] ** -0.5).masked_fill(
                torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
            out.append((s.softmax(-1) @ c).transpose(0, 1))
            at += n
        return torch.cat(out + [torch.zeros(q.shape[0] - at, *q.shape[1:], dtype=q.dtype, device="cuda")])

    def ffn(self, x, w1, w3, w2):
        g = x @ w1
        return (g * torch.sigmoid(g) * (x @ w3)) @ w2


@pytest.mark.parametrize("captured", [False, True])
def test_a_decoder_block_forward_and_backward(captured):
    """All of it together under autograd, eager and captured, against 64 bits.  About fifteen tensors in a row are rounded to bf16 on the
    way of every entry, most of them beside a stream that is larger: within 15 roundings of 2^-8 in the root mean
    square."""
    torch.manual_seed(0)
    lengths, T, d, F, V, dim, heads = [130, 64, 0, 201], 400, 128, 352, 40, 64, (4, 2, 2)
    side = torch.cuda.Stream()
    owner = binding.Context("cuda:0", stream=side if captured else None)
    seq = binding.Sequences(owner, lengths, T)
    seq.positions
    shapes = dict(embed=(V, d), wq=(d, 4 * dim), wk=(d, 2 * dim), wv=(d, 2 * dim), wo=(4 * dim, d), w1=(d, F), w3=(d, F), w2=(F, d))
    p = {n: (torch.randn(*s, device="cuda") * s[0] ** -0.5).to(BF16).requires_grad_() for n, s in shapes.items()}
    p.update({n: (1 + 0.1 * torch.randn(d, device="cuda")).requires_grad_() for n in ("g1", "g2", "g3")})
    ids = torch.randint(0, V, (T,), device="cuda")
    ang = torch.arange(256, device="cuda")[:, None] * 100.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))
    cos, sin = ang.cos(), ang.sin()
    weight = torch.randn(T, d, device="cuda").to(BF16)
    weight[sum(lengths):] = 0                # tokens of no sequence have no loss

    def step():
        y = block(Library(owner), p, ids, seq, cos, sin, heads)
        return [y, *torch.autograd.grad(y, list(p.values()), weight)]

    if captured:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
        graph.replay()
        torch.cuda.synchronize()
    else:
        got = step()
    owner.sync_status()
    p64 = {n: t.detach().double().requires_grad_() for n, t in p.items()}
    y = block(Definition(), p64, ids, seq, cos, sin, heads)
    want = [y, *torch.autograd.grad(y, list(p64.values()), weight.double())]
    used = sum(lengths)
    for name, a, b in zip(("y", *p), got, want):
        a, b = a.detach().double(), b.detach()
        if name == "y":
            a, b = a[:used], b[:used]
        assert torch.isfinite(a).all(), name
        assert (a - b).norm() <= 15 * 2.0 ** -8 * b.norm(), (name, float((a - b).norm() / b.norm()))
    if captured:
        del graph, got
    owner.close()
