"""The operators in the framework's own path: 8-bit AdamW states inside the MuLoCo inner step, the autograd
forms, and the example that trains a small model with all of them."""
import dataclasses
import importlib.util
import os

import numpy as np
import pytest

from paper_2505_23725_b200 import configs, synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _workload(bits, **kw):
    return configs.mini_workload(K=2, H=2, vocab=100, norms=True, adam_state_bits=bits, **kw)


def _grads(w, seed):
    import torch
    rng = np.random.default_rng(seed)
    return [[torch.from_numpy(g).cuda() for g in synth.host_gradients(rng, w.tensors)] for _ in range(w.K)]


def test_inner_step_with_8_bit_states_equals_the_list_operator():
    import torch
    from paper_2505_23725_b200 import binding
    w = _workload(8)
    init = synth.init_weights(np.random.default_rng(1), w.tensors)
    opt = binding.MuLoCo(w, "cuda:0", init=init)
    one = binding.MuLoCo(w, "cuda:0", init=init)                 # the same steps, one worker at a time
    ids = [i for i, t in enumerate(w.tensors) if t.kind == configs.ADAMW]
    ctx = binding.Context("cuda:0")
    lists, params = [], []
    for k in range(w.K):
        p = [opt.theta_k[k][i].clone() for i in ids]
        params.append(p)
        lists.append(binding.AdamW(ctx, p, lr=w.muon_lr, beta1=w.adam_beta1, beta2=w.adam_beta2, eps=w.adam_eps,
                                   weight_decay=w.muon_wd, state_bits=8, seed=k, wd_mult=[w.tensors[i].wd_mult for i in ids]))
    for step in range(4):
        g = _grads(w, step)
        opt.inner_step(-1, g, lr_scale=0.5 + step)
        for k in reversed(range(w.K)):
            one.inner_step(k, g[k], lr_scale=0.5 + step)
            lists[k].step([g[k][i] for i in ids], lr_scale=0.5 + step)
        for k in range(w.K):
            m, v = lists[k].moments()
            for j, i in enumerate(ids):
                assert torch.equal(opt.theta_k[k][i], params[k][j]) and torch.equal(one.theta_k[k][i], params[k][j])
                a, b = opt.adam_moments(k, i)
                o, n = lists[k].offsets[j], w.tensors[i].numel
                assert torch.equal(a.reshape(-1), m[o:o + n]) and torch.equal(b.reshape(-1), v[o:o + n])
                assert torch.equal(opt.state1[k][i], one.state1[k][i]) and torch.equal(opt.state2[k][i], one.state2[k][i])
    # the hidden matrices know nothing of it
    full = binding.MuLoCo(dataclasses.replace(w, adam_state_bits=32), "cuda:0", init=init)
    for step in range(4):
        full.inner_step(-1, _grads(w, step), lr_scale=0.5 + step)
    for i, t in enumerate(w.tensors):
        if t.kind == configs.MUON:
            assert torch.equal(full.theta_k[1][i], opt.theta_k[1][i]) and torch.equal(full.state1[1][i], opt.state1[1][i])
        else:                                                    # and 8 bits stay near 32: a step is about lr * 5
            d = (full.theta_k[1][i] - opt.theta_k[1][i]).norm() / (full.theta_k[1][i] - full.theta_g[i]).norm()
            assert d < 0.1, (t.name, float(d))
    opt.outer_sync(-1)
    opt.sync_status()
    full.sync_status()
    assert opt.get_timings()[1] > 0
    for o in lists + [opt, one, full, ctx]:
        o.close()


def test_8_bit_states_from_host_gradients_and_resumed():
    import torch
    from paper_2505_23725_b200 import binding
    w = _workload(8, ns_mode="bf16")
    init = synth.init_weights(np.random.default_rng(2), w.tensors)
    a, b, c = (binding.MuLoCo(w, "cuda:0", init=init) for _ in range(3))
    for step in range(4):
        g = _grads(w, 10 + step)
        a.inner_step(-1, g)
        b.inner_step_host(-1, [[x.cpu().pin_memory() for x in gk] for gk in g])
        b.sync_status()
        if step == 1:                                            # a checkpoint: the tensors and the small host state
            for k in range(w.K):
                for i in range(len(w.tensors)):
                    c.theta_k[k][i].copy_(a.theta_k[k][i])
                    c.state1[k][i].copy_(a.state1[k][i])
                    if a.state2[k][i] is not None:
                        c.state2[k][i].copy_(a.state2[k][i])
            c.set_state(a.get_state())
        if step > 1:
            c.inner_step(-1, g)
    a.sync_status()
    for k in range(w.K):
        for i in range(len(w.tensors)):
            assert torch.equal(a.theta_k[k][i], b.theta_k[k][i]) and torch.equal(a.theta_k[k][i], c.theta_k[k][i])
            assert torch.equal(a.state1[k][i], c.state1[k][i])
    for o in (a, b, c):
        o.close()


def test_8_bit_states_refusals():
    from paper_2505_23725_b200 import binding
    with pytest.raises(binding.MulocoError) as e:
        binding.MuLoCo(_workload(16), "cuda:0")
    assert e.value.status == binding.EINVAL and "adam_state_bits" in str(e.value)


def test_autograd_forms():
    """The gradients that autograd hands out are those of the operators, and differences of the loss agree with them."""
    import torch
    from paper_2505_23725_b200 import binding, layers
    ctx = binding.Context("cuda:0")
    torch.manual_seed(0)
    bf = torch.bfloat16
    x = torch.randn(2, 9, 64, device="cuda").to(bf).requires_grad_()
    ws = [(torch.randn(*s, device="cuda") / 8).to(bf).requires_grad_() for s in ((64, 136), (64, 136), (136, 64))]
    dy = torch.randn(2, 9, 64, device="cuda").to(bf)
    y = layers.gated_ffn(ctx, x, *ws, activation="gelu")
    y.backward(dy)
    y0, saved = ctx.gated_ffn(x.detach().view(18, 64), *(t.detach() for t in ws), "gelu")
    want = ctx.gated_ffn_backward(dy.view(18, 64), x.detach().view(18, 64), *(t.detach() for t in ws), saved, "gelu")
    assert torch.equal(y.detach().view(18, 64), y0) and torch.equal(x.grad.view(18, 64), want[0])
    assert all(torch.equal(t.grad, g) for t, g in zip(ws, want[1:]))
    with torch.no_grad():
        assert torch.equal(layers.gated_ffn(ctx, x, *ws, activation="gelu"), y)

    q, k = (torch.randn(7, h, 16, device="cuda", requires_grad=True) for h in (3, 1))
    gq, gk = (torch.ones(16, device="cuda").requires_grad_() for _ in range(2))
    ang = torch.randn(7, 8, device="cuda")
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    def loss(q_, k_, a, b):
        u, v = layers.qk_norm_rope(ctx, q_, k_, ang.cos(), ang.sin(), None, a, b)
        return (u * dq).sum() + (v * dk).sum()
    loss(q, k, gq, gk).backward()
    # a central difference of step 1e-2 along a random direction, float32: rounding of the loss (about 1e-5 of it) over
    # 2e-2, truncation 1e-4 of the third derivative
    for t in (q, k, gq, gk):
        v = torch.randn_like(t)
        args = [s.detach() for s in (q, k, gq, gk)]
        j = next(n for n, s in enumerate((q, k, gq, gk)) if s is t)
        up, down = list(args), list(args)
        up[j], down[j] = args[j] + 1e-2 * v, args[j] - 1e-2 * v
        num = (loss(*up) - loss(*down)).item() / 2e-2
        assert abs(num - (t.grad * v).sum().item()) < 2e-2 * max(1.0, t.grad.norm().item() * v.norm().item() / 10)
    ctx.sync_status()
    ctx.close()


def test_example_learns():
    spec = importlib.util.spec_from_file_location("train_tiny_lm", os.path.join(ROOT, "examples", "train_tiny_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.train(rounds=6, quiet=True)
    assert all(np.isfinite(losses))
    # the text's entropy is 1.76 a token (next token by the table with probability 0.752, 127 others with 0.00195 each), below
    # which no model gets; uniform guessing is ln 128 = 4.85; 10 steps of 4096 tokens show every pair some 300 times
    assert losses[-1] < losses[0] < 4.85 and 1.7 < losses[-1] < 2.0, losses
