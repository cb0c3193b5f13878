"""Causal attention over packed sequences on the GPU, against the definition in 64 bits.

Tolerances, per element, count roundings (bf16: 2^-8 of the value).  o: the weights p are rounded as an operand, the
result is rounded: 2^-8 (sum_j p |v| + |o|).  dv likewise with do.  dq, dk: ds is rounded, and delta = do . o uses the
rounded o: 2^-8 (sum |ds| |k| + sum p |k| sum_d |do o| + |result|).  Float32 sums and the hardware's exponential are far below
that: another 2^-6 of the bound, and the scores' own error (D 2^-23 of the sum of their terms' magnitudes, at most)
relative to every weight.  lse: the scores' error and 2^-20 of one plus its size (exponential, logarithm, sum)."""
import pytest
import torch

from paper_2505_23725_b200 import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context("cuda:0")
    yield c
    c.sync_status()
    c.close()


def inputs(lengths, tail, hq, hk, D, layout="dense", seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lengths) + tail

    def rand(*shape, s=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * s).to(torch.bfloat16)

    if layout == "fused":                    # views of one projection's rows
        qkv = rand(T, hq + 2 * hk, D, s=spread)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    elif layout == "heads first":
        q, k, v = (rand(h, T, D, s=spread).transpose(0, 1) for h in (hq, hk, hk))
    else:
        q, k, v = rand(T, hq, D, s=spread), rand(T, hk, D, s=spread), rand(T, hk, D, s=spread)
    return q, k, v, rand(T, hq, D)


def reference(q, k, v, do, lengths, scale):
    """Results and gradients in 64 bits, and the tolerance of each."""
    T, hq, D = q.shape
    hk = k.shape[1]
    group = hq // hk
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=q.device)          # noqa: E731
    r = {"o": z(T, hq, D), "lse": z(hq, T), "dq": z(T, hq, D), "dk": z(T, hk, D), "dv": z(T, hk, D)}
    tol = {n: torch.zeros_like(t) for n, t in r.items()}
    a = 0
    for n in lengths:
        b = a + n
        if n == 0:
            continue
        later = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
        for h in range(hq):
            Q, K, V, G = q[a:b, h].double(), k[a:b, h // group].double(), v[a:b, h // group].double(), do[a:b, h].double()
            s = (Q @ K.T * scale).masked_fill(later, -torch.inf)
            lse = torch.logsumexp(s, 1)
            p = (s - lse[:, None]).exp()
            o = p @ V
            off = D * 2.0 ** -23 * scale * (Q.abs() @ K.abs().T).masked_fill(later, 0.0)      # of a score
            err = off + off.amax(1, keepdim=True) + 2.0 ** -20                                # of a weight, relative
            r["o"][a:b, h], r["lse"][h, a:b] = o, lse
            tol["o"][a:b, h] = U * (1 + 2.0 ** -6) * (p @ V.abs() + o.abs()) + (p * err) @ V.abs()
            tol["lse"][h, a:b] = off.amax(1) + 2.0 ** -20 * (1 + lse.abs())
            dp = G @ V.T
            delta = (G * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            slack = U * (1 + 2.0 ** -6) * (ds.abs() + p * (G * o).abs().sum(1, keepdim=True)) \
                + p * (err + 2.0 ** -20) * (dp.abs() + delta.abs() + G.abs() @ V.abs().T)
            r["dq"][a:b, h] = scale * ds @ K
            tol["dq"][a:b, h] = scale * slack @ K.abs() + U * (scale * ds @ K).abs()
            r["dk"][a:b, h // group] += scale * ds.T @ Q
            tol["dk"][a:b, h // group] += scale * slack.T @ Q.abs()
            r["dv"][a:b, h // group] += p.T @ G
            tol["dv"][a:b, h // group] += U * (1 + 2.0 ** -6) * p.T @ G.abs() + (p * err).T @ G.abs()
        a = b
    for n in ("dk", "dv"):
        tol[n] += U * (1 + 2.0 ** -6) * r[n].abs()
    return r, tol


def check(got, r, tol, name):
    got = got.double()
    assert torch.isfinite(got).all(), name
    excess = (got - r[name]).abs() - tol[name] - 1e-30
    assert excess.max() <= 0, f"{name}: {int((excess > 0).sum())} of {excess.numel()} beyond the tolerance"


def run(ctx, q, k, v, do, lengths, scale=None):
    seq = binding.Sequences(ctx, lengths, tokens=q.shape[0])
    o, lse = ctx.causal_attention(q, k, v, seq, scale=scale)
    real = q.shape[2] ** -0.5 if scale is None else scale
    r, tol = reference(q, k, v, do, lengths, real)
    check(o, r, tol, "o")
    check(lse, r, tol, "lse")
    # the backward pass on its own: from the reference's o and lse
    grads = ctx.causal_attention_backward(do, q, k, v, r["o"].to(torch.bfloat16), r["lse"].float(), seq, scale=scale)
    for n, t in zip(("dq", "dk", "dv"), grads):
        check(t, r, tol, n)
    ctx.sync_status()
    return (o, lse) + grads


CASES = [
    ([1], 0, 1, 1, 64, "dense"),
    ([1], 0, 12, 12, 64, "fused"),
    ([2, 1, 3], 0, 2, 1, 128, "dense"),
    ([127], 0, 2, 2, 64, "dense"),
    ([128], 0, 2, 2, 128, "fused"),
    ([129], 1, 2, 1, 128, "heads first"),
    ([255, 1, 257], 5, 4, 2, 64, "fused"),
    ([256, 0, 384], 130, 3, 3, 128, "dense"),
    ([385, 500, 0, 77], 0, 6, 2, 80, "fused"),
    ([40, 300, 0, 0], 300, 8, 1, 8, "dense"),
    ([700], 0, 2, 1, 40, "heads first"),
    ([1030, 90], 3, 4, 4, 112, "dense"),
    ([5] * 30 + [130], 0, 2, 2, 32, "fused"),
    ([2100], 17, 2, 1, 128, "dense"),
    ([1600, 600], 0, 6, 2, 64, "fused"),
]


@pytest.mark.parametrize("lengths,tail,hq,hk,D,layout", CASES, ids=lambda x: str(x).replace(" ", "")[:24])
def test_against_64_bits(ctx, lengths, tail, hq, hk, D, layout):
    q, k, v, do = inputs(lengths, tail, hq, hk, D, layout)
    out = run(ctx, q, k, v, do, lengths)
    if tail:                                 # tokens of no sequence
        o, lse, dq, dk, dv = out
        assert all(not t[-tail:].any() for t in (o, dq, dk, dv)) and not lse[:, -tail:].any()


@pytest.mark.parametrize("scale,spread", [(1.0, 0.3), (0.02, 3.0), (0.125, 6.0), (1e-6, 1.0)])
def test_scales_and_sharp_weights(ctx, scale, spread):
    """Flat weights, and scores far apart, whose maximum moves from tile to tile."""
    q, k, v, do = inputs([700, 130], 0, 3, 1, 64, spread=spread, seed=4)
    run(ctx, q, k, v, do, [700, 130], scale=scale)


def test_growing_maximum(ctx):
    """Scores that rise along the keys: the maximum moves at every tile."""
    q, k, v, do = inputs([900], 0, 2, 2, 64, seed=5)
    k = (k.float() * torch.linspace(0.1, 8.0, 900, device="cuda")[:, None, None]).to(torch.bfloat16)
    run(ctx, q, k, v, do, [900], scale=0.5)
