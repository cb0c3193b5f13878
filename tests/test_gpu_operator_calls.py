"""Calls of the operators on a B200: what they allocate, calls inside a captured graph, calls from several threads."""
import pytest

pytestmark = pytest.mark.gpu


def _qk(D=64, T=300, seed=0):
    import torch
    torch.manual_seed(seed)
    q, k, dq, dk = (torch.randn(T, h, D, device="cuda") for h in (4, 2, 4, 2))
    cos, sin = torch.randn(T, D // 2, device="cuda"), torch.randn(T, D // 2, device="cuda")
    gq, gk = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    return (dq, dk, q, k, cos, sin, None, gq, gk), (q, k, cos, sin, None, gq, gk)


def test_first_norm_backward_of_a_context_allocates_nothing():
    import torch
    from paper_2505_23725_b200 import binding
    back, fwd = _qk()
    warm = binding.Context("cuda:0")               # kernels loaded, torch's blocks cached
    want = warm.qk_norm_rope_backward(*back)
    del want
    ctx = binding.Context("cuda:0")
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    got = ctx.qk_norm_rope_backward(*back)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
    want = warm.qk_norm_rope_backward(*back)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for c in (ctx, warm):
        c.sync_status()
        c.close()


def test_operators_inside_a_captured_graph():
    """A fresh context's calls, captured and replayed on other values, give what they give outside a graph."""
    import torch
    from paper_2505_23725_b200 import binding
    plain = binding.Context("cuda:0")
    back, fwd = _qk()
    T, d, F = 200, 64, 136
    x, dy = (torch.randn(T, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    w1, w3 = (torch.randn(d, F, device="cuda").to(torch.bfloat16) / 8 for _ in range(2))
    w2 = torch.randn(F, d, device="cuda").to(torch.bfloat16) / 8

    def calls(c):
        y, saved = c.gated_ffn(x, w1, w3, w2)
        return [*c.qk_norm_rope(*fwd), *c.qk_norm_rope_backward(*back), y, *c.gated_ffn_backward(dy, x, w1, w3, w2, saved)]

    calls(plain)
    side = torch.cuda.Stream()
    ctx = binding.Context("cuda:0", stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = calls(ctx)
    for seed in (1, 2):
        torch.manual_seed(seed)
        for t in (*back[:4], x, dy):
            t.copy_(torch.randn(t.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, calls(plain)))
    plain.sync_status()
    ctx.sync_status()
    del graph
    ctx.close()
    plain.close()


def test_calls_from_several_threads_with_sizes_in_turn():
    """Gain gradients are summed in an order that the grid fixes: with other head sizes on their way in other threads it has to
    be the same grid, hence the same bits."""
    import threading
    import torch
    from paper_2505_23725_b200 import binding
    sizes = (64, 128, 96, 32)
    inputs = {D: _qk(D, 3000, seed=D)[0] for D in sizes}
    ctx = binding.Context("cuda:0")
    want = {D: ctx.qk_norm_rope_backward(*inputs[D]) for D in sizes}
    x = torch.randn(40, 64, device="cuda").to(torch.bfloat16)
    w = torch.randn(64, 64, device="cuda").to(torch.bfloat16) / 8
    y = ctx.gated_ffn(x, w, w, w)[0]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            mine = binding.Context("cuda:0", stream=stream)
            for n in range(60):
                D = sizes[(i + n) % len(sizes)]
                got = mine.qk_norm_rope_backward(*inputs[D])
                if not all(torch.equal(a, b) for a, b in zip(got, want[D])):
                    wrong.append((i, n, D))
                if not torch.equal(mine.gated_ffn(x, w, w, w)[0], y):
                    wrong.append((i, n, "ffn"))
            mine.sync_status()
            mine.close()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    ctx.close()


@pytest.mark.parametrize("shape", [(5, 64, 136), (100, 264, 520), (300, 128, 264), (900, 1024, 1160), (4100, 1032, 1160)], ids=str)
@pytest.mark.parametrize("back", [False, True])
def test_a_wait_that_runs_out_is_reported_and_the_context_stays_usable(shape, back):
    """One thread block issues no copies: the waits for them run out after the 2 ms that the test sets, the kernel returns, the timeout is
    reported once, and the next call is right.  Few-token and 256 x 256 forms; with 128 or fewer columns of X the other CTA of the
    pair has issued all its copies, and its copying thread is done, long before a wait runs out."""
    import time
    import torch
    from paper_2505_23725_b200 import binding
    T, d, F = shape
    torch.manual_seed(T)
    bf = torch.bfloat16
    x, dy = (torch.randn(T, d, device="cuda").to(bf) for _ in range(2))
    w1, w3 = ((torch.randn(d, F, device="cuda") * d ** -0.5).to(bf) for _ in range(2))
    w2 = (torch.randn(F, d, device="cuda") * F ** -0.5).to(bf)
    ctx = binding.Context("cuda:0")
    _, saved = ctx.gated_ffn(x, w1, w3, w2)

    def call():
        if back:
            return ctx.gated_ffn_backward(dy, x, w1, w3, w2, saved)
        out, kept = ctx.gated_ffn(x, w1, w3, w2)
        return (out, *kept)
    want = call()
    ctx.sync_status()
    def hook(what, value):
        assert ctx.lib.muloco_debug_set(ctx.ctx, what, value) == binding.OK
    hook(binding.DEBUG_WAIT_LIMIT_NS, 2_000_000)
    hook(binding.DEBUG_WITHHOLD_COPY, 1)
    t0 = time.perf_counter()
    call()
    with pytest.raises(binding.MulocoError) as e:
        ctx.sync_status()
    assert e.value.status == binding.ETIMEOUT
    assert time.perf_counter() - t0 < 5.0
    ctx.sync_status()                                   # read once
    hook(binding.DEBUG_WAIT_LIMIT_NS, 0)
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    ctx.sync_status()
    ctx.close()


def test_autograd_forms_take_any_layout():
    """layers.py in front of the library itself: inputs and gradients whose layout it refuses give the bits of contiguous ones."""
    import torch
    from paper_2505_23725_b200 import binding, layers
    ctx = binding.Context("cuda:0")
    torch.manual_seed(0)
    T, d, F, bf = 70, 64, 136, torch.bfloat16
    x, other = (torch.randn(T, d, device="cuda").to(bf) for _ in range(2))
    ws = [(torch.randn(*s, device="cuda") / 8).to(bf) for s in ((d, F), (d, F), (F, d))]
    wide = torch.cat([other[:, :1], x, other[:, :2]], 1)
    row = torch.randn(d, device="cuda").to(bf)
    losses = (lambda y: (y.sum(0) * row).sum(), lambda y: (torch.cat([y, other[:, :3]], 1) * wide).float().sum(),
              lambda y: (torch.cat([other[:, :3], y], 1) * wide).float().sum(), lambda y: (y * other).float().sum())
    # the gradients that reach the block, contiguous
    for loss in losses:
        y0 = torch.zeros(T, d, dtype=bf, device="cuda", requires_grad=True)
        dy = torch.autograd.grad(loss(y0), y0)[0].contiguous()
        want = ctx.gated_ffn_backward(dy, x, *ws, ctx.gated_ffn(x, *ws)[1])
        for view in (x, wide[:, 1:d + 1], x.t().contiguous().t()):
            leaves = [t.detach().requires_grad_() for t in (view, *ws)]
            loss(layers.gated_ffn(ctx, *leaves)).backward()
            assert all(torch.equal(t.grad, g) for t, g in zip(leaves, want))
    q = torch.randn(9, 3, 16, device="cuda", requires_grad=True)
    gain, ang = torch.randn(16, device="cuda", requires_grad=True), torch.randn(9, 8, device="cuda")
    dq = torch.randn(9, 16, 3, device="cuda").transpose(1, 2)
    want = ctx.qk_norm_rope_backward(dq.contiguous(), None, q.detach(), None, ang.cos(), ang.sin(), None, gain.detach())
    for alone in (0, 1):
        pair, gains = [None, None], [None, None]
        pair[alone], gains[alone] = q, gain
        out = layers.qk_norm_rope(ctx, *pair, ang.cos(), ang.sin(), None, *gains)
        assert out[1 - alone] is None
        got = torch.autograd.grad(out[alone], (q, gain), dq)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[2])
    ctx.sync_status()
    ctx.close()


def test_other_threads_run_while_a_call_waits():
    """A launch into a full queue waits for the GPU, which may itself wait for a Python callback: the compiled call path does not hold
    the interpreter meanwhile.  A C function that sleeps for as many microseconds as its first argument says stands in for the library's."""
    import ctypes
    import threading
    import time
    import torch
    from paper_2505_23725_b200 import _fastcall
    libc = ctypes.CDLL(None)
    sleep = ctypes.cast(libc.usleep, ctypes.c_void_p).value
    stream = torch.cuda.current_stream(0).cuda_stream
    _fastcall.adamw_step(1, sleep, 0, stream, 1, 1.0)
    ticks, stop = [0], threading.Event()

    def tick():
        while not stop.is_set():
            ticks[0] += 1
            time.sleep(0.001)

    t = threading.Thread(target=tick)
    t.start()
    time.sleep(0.05)
    before = ticks[0]
    t0 = time.perf_counter()
    r = _fastcall.adamw_step(400_000, sleep, 0, stream, 1, 1.0)
    took, during = time.perf_counter() - t0, ticks[0] - before
    stop.set()
    t.join()
    assert r == 0 and took > 0.3
    assert during > 20, during
