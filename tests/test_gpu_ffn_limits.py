"""The feed-forward block at the ends of bf16's range."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

GATES = [0.0, 1.0, -1.0, 9.0, -9.0, 88.0, -88.0, 1e3, -1e3, 1e7, -1e7, 3e13, -3e13, 1e20, -1e20, 3e38, -3e38]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [1, 700, 900])     # either form of the kernel that makes dG and dU
def test_gate_gradient_of_large_gates(act, T):
    """Any finite G: act'(G) is 1 or 0 far from zero, and no NaN.  dY and W2 make dH = 1 in every entry, U = 1, so dG = act'(G) and
    dU = act(G), each rounded once; they are read off dW1 and dW3 with X = 1 in one token."""
    import torch
    from paper_2505_23725_b200 import binding
    ctx = binding.Context("cuda:0")
    d, F, bf = 1024, 1160, torch.bfloat16
    row = torch.tensor(GATES, dtype=torch.float64).to(bf)
    g = row.repeat(F // len(GATES) + 1)[:F].expand(T, F).contiguous().cuda()
    u = torch.ones(T, F, dtype=bf, device="cuda")
    x, dy = torch.zeros(T, d, dtype=bf, device="cuda"), torch.zeros(T, d, dtype=bf, device="cuda")
    x[T // 2, 0], dy[:, 3] = 1.0, 1.0
    w2 = torch.zeros(F, d, dtype=bf, device="cuda")
    w2[:, 3] = 1.0
    w = torch.zeros(d, F, dtype=bf, device="cuda")
    dx, dw1, dw3, _ = ctx.gated_ffn_backward(dy, x, w, w, w2, (g, u, u), activation=act)
    ctx.sync_status()
    # in 64 bits with the logistic function (1 + tanh loses what is left of it at G = -9), clipped where nothing is left in 64 either
    G = g[0].double().cpu().numpy()
    c = np.clip(G, -100.0, 100.0)
    k = 2 * np.sqrt(2 / np.pi)
    p, dp = (c, 1.0) if act == "silu" else (k * (c + 0.044715 * c ** 3), k * (1 + 3 * 0.044715 * c * c))
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-p))
    value = np.where(G < -100, 0.0, G * s)
    slope = s + c * dp * s * (1 - s)
    for got, want, name in ((dw1[0], slope, "act'"), (dw3[0], value, "act")):
        got = got.double().cpu().numpy()
        # one bf16 rounding (2^-8) and the approximations' few units; below 1e-30 only that it is as small
        ok = np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-5 * np.abs(want) + 1e-30
        assert ok.all(), (name, act, [(G[i], got[i], want[i]) for i in np.flatnonzero(~ok)[:4]])
    assert not dw1[1:].any() and not dw3[1:].any() and torch.isfinite(dx.float()).all()
    ctx.close()
