"""AdamW states on the GPU: blocks of 8-bit states after a value that is not finite, states made on another stream."""
import pytest

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def ctx():
    from paper_2505_23725_b200 import binding
    c = binding.Context("cuda:0")
    yield c
    c.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -1e25])      # (the square of the last is beyond float32)
@pytest.mark.parametrize("at", [700, 999])                                  # inside a whole block, and in the short last one
def test_8_bit_block_stays_nan_and_is_reported_every_step(ctx, value, at, bf16):
    """The scales that a block's elements share turn NaN, so by the formulas its moments are NaN at every later step and its
    parameters from the next one on; each step says so, and the other blocks know nothing of it."""
    import torch
    from paper_2505_23725_b200 import binding
    n, blk = 1000, at // 256
    dt = torch.bfloat16 if bf16 else torch.float32
    torch.manual_seed(0)
    grads = [(torch.randn(n, device="cuda") * 1e-2).to(dt) for _ in range(4)]
    hit = [g.clone() for g in grads]
    hit[1][at] = value
    p, q = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    good = binding.AdamW(ctx, [p], state_bits=8, seed=3, grad_dtype=dt, **HYPER)
    bad = binding.AdamW(ctx, [q], state_bits=8, seed=3, grad_dtype=dt, **HYPER)
    inside = torch.arange(n, device="cuda") // 256 == blk
    for t in range(4):
        good.step([grads[t]])
        ctx.sync_status()
        bad.step([hit[t]])
        if t == 0:
            ctx.sync_status()
            assert torch.equal(p, q)
            continue
        with pytest.raises(binding.MulocoError) as e:
            ctx.sync_status()
        assert e.value.status == binding.ENONFINITE
        assert torch.isnan(bad.scale1[blk]) and torch.isnan(bad.scale2[blk])
        m, v = bad.moments()
        assert torch.isnan(m[:n][inside]).all() and torch.isnan(v[:n][inside]).all()
        if t > 1:
            assert torch.isnan(q[inside]).all()
        m0, v0 = good.moments()
        assert torch.equal(q[~inside], p[~inside])
        assert torch.equal(m[:n][~inside], m0[:n][~inside]) and torch.equal(v[:n][~inside], v0[:n][~inside])
        others = torch.arange(4, device="cuda") != blk
        assert torch.equal(bad.scale1[others], good.scale1[others]) and torch.equal(bad.scale2[others], good.scale2[others])
    good.close()
    bad.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_list_built_on_a_busy_stream(bits):
    """States made on a stream that is still at work, first step on the context's: it finds them zero."""
    import torch
    from paper_2505_23725_b200 import binding
    n = 1 << 20
    torch.manual_seed(0)
    g = torch.randn(n, device="cuda")
    own, busy = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = binding.Context("cuda:0", stream=own)
    torch.cuda.synchronize()
    outs = []
    for late in (False, True):
        p = torch.ones(n, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(busy if late else own):
            # what the states' memory holds before
            old = [torch.full((k * n,), 85, dtype=torch.uint8, device="cuda") for k in (1, 1, 4, 4)] + \
                  [torch.full((n // 256,), 3.0, device="cuda") for _ in range(2)]
            torch.cuda.synchronize()
            del old
            if late:
                big = torch.randn(8192, 8192, device="cuda")
                for _ in range(20):
                    big = big @ big * 1e-2
            opt = binding.AdamW(ctx, [p], state_bits=bits, seed=1, **HYPER)
        with torch.cuda.stream(own):
            opt.step([g])
        torch.cuda.synchronize()
        outs.append([p] + [t.clone() for t in (opt.state1, opt.state2, opt.scale1, opt.scale2) if t is not None])
        opt.close()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    ctx.sync_status()
    ctx.close()


def test_optimizer_built_on_a_busy_stream():
    """The same for a MuLoCo with a stream of its own: its replicas start from the global parameters."""
    import torch
    from paper_2505_23725_b200 import binding, configs
    w = configs.mini_workload(K=2, H=2, vocab=100, norms=True, adam_state_bits=8)
    own, busy = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(busy):
        big = torch.randn(8192, 8192, device="cuda")
        torch.cuda.synchronize()
        for _ in range(20):
            big = big @ big * 1e-2
        opt = binding.MuLoCo(w, "cuda:0", init_seed=3, stream=own)
    torch.cuda.synchronize()
    for i in range(len(w.tensors)):
        assert torch.equal(opt.theta_k[0][i], opt.theta_g[i]) and torch.equal(opt.theta_k[1][i], opt.theta_g[i])
        assert opt.theta_g[i].any()
    opt.sync_status()
    opt.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [8, 32])
def test_inner_step_refuses_a_misaligned_gradient_before_it_changes_anything(bits, dtype):
    import ctypes as C
    import torch
    from paper_2505_23725_b200 import binding, configs
    w = configs.mini_workload(K=2, H=2, vocab=100, norms=True, adam_state_bits=bits, grad_dtype=dtype)
    opt = binding.MuLoCo(w, "cuda:0", init_seed=1, alloc_grads=True)
    for g in opt.flat_grads:
        g.normal_()
    opt.inner_step()
    opt.sync_status()

    def state():
        return [t.clone() for per in (opt.theta_k, opt.state1, opt.state2) for k in range(w.K) for t in per[k] if t is not None]

    before, blob = state(), opt.get_state()
    last = max(i for i, t in enumerate(w.tensors) if t.kind == configs.ADAMW)
    ptrs = [opt.grads[k][i].data_ptr() for k in range(w.K) for i in range(opt.n)]
    ptrs[opt.n + last] += 1 if dtype == "bf16" else 2
    table = (C.c_void_p * len(ptrs))(*ptrs)
    assert opt.lib.muloco_inner_step(opt.ctx, -1, table, 1.0) == binding.EINVAL
    assert b"aligned" in opt.lib.muloco_last_error(opt.ctx)
    opt.sync_status()
    assert all(torch.equal(a, b) for a, b in zip(before, state())) and opt.get_state() == blob
    opt.inner_step()
    opt.sync_status()
    opt.close()


def test_workers_spread_over_contexts_round_as_in_one():
    """8-bit states: the dither goes by the worker's number in the whole run, so two contexts of one worker each give what
    one context of two gives; with the same number they would round alike."""
    import dataclasses
    import torch
    from paper_2505_23725_b200 import binding, configs
    w = configs.mini_workload(K=2, H=2, vocab=100, norms=True, adam_state_bits=8)
    both = binding.MuLoCo(w, "cuda:0", init_seed=1, alloc_grads=True)
    one = [binding.MuLoCo(dataclasses.replace(w, K=1, adam_seed=s), "cuda:0", init_seed=1, alloc_grads=True) for s in (0, 1)]
    for step in range(3):
        torch.manual_seed(step)
        both.flat_grads[0].normal_()
        both.flat_grads[1].copy_(both.flat_grads[0])              # the same gradients: only the dither differs
        for o in one:
            o.flat_grads[0].copy_(both.flat_grads[0])
            o.inner_step()
        both.inner_step()
    for i, t in enumerate(w.tensors):
        for k in range(2):
            assert torch.equal(both.theta_k[k][i], one[k].theta_k[0][i])
            assert torch.equal(both.state1[k][i], one[k].state1[0][i])
            if t.kind == configs.ADAMW:
                assert torch.equal(both.state2[k][i], one[k].state2[0][i])
        if t.kind == configs.ADAMW:
            assert not torch.equal(both.state1[0][i], both.state1[1][i])
    for o in (both, *one):
        o.sync_status()
        o.close()
