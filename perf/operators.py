"""Measured cases of the operators around the optimizer step: AdamW over many tensors (states in 8 or 32 bits),
the per-head norm of queries and keys with the position rotation, and the gated feed-forward block, the last two
forward and backward.

`run` computes an operator in its plain form (elementary torch operations in 32 bits, rounded once at the end) or,
with `own` set, through the library.  Sizes are those of the benchmark configurations (widths 768 / 1024 / 2048,
feed-forward widths 2048 / 2816 / 5632, vocabulary 32000, sequences of 2048) and odd ones around them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BLOCK = 256                                  # elements that share a scale in the 8-bit states
BF16, F32 = torch.bfloat16, torch.float32


def f32(x):
    """The value of x as the library holds it (32 bits)."""
    return float(np.float32(x))


ADAM = dict(lr=f32(1e-2), beta1=f32(0.9), beta2=f32(0.99), eps=f32(1e-8), weight_decay=f32(6.25e-4))
ADAM_SEED, ADAM_STEPS = 1234, 700            # seed of the dither; steps behind the states that prepare() makes
EPS = f32(1e-6)


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest step: the 25 norm gains of the 12-layer, 768-wide model, 32-bit states; latency
        dict(name="adamw32 gains", op="adamw", tensors="gains", layers=12, d=768, F=2048, vocab=32000, bits=32,
             grad="f32", copy=False),
        # what AdamW keeps in MuLoCo: embedding, head and gains of that model; 8-bit states, bf16 gradients,
        # bf16 working copy of the parameters for the next forward pass
        dict(name="adamw8 rest 768", op="adamw", tensors="rest", layers=12, d=768, F=2048, vocab=32000, bits=8,
             grad="bf16", copy=True),
        # the DiLoCo baseline (AdamW on every tensor) at width 768, 32-bit states, bf16 gradients
        dict(name="adamw32 all 768", op="adamw", tensors="all", layers=12, d=768, F=2048, vocab=32000, bits=32,
             grad="bf16", copy=False),
        # the DiLoCo baseline at width 1024, 24 layers, 8-bit states, f32 gradients: the largest
        dict(name="adamw8 all 1024", op="adamw", tensors="all", layers=24, d=1024, F=2816, vocab=32000, bits=8,
             grad="f32", copy=False),
        # one new token of a 768-wide model with 12 heads: latency
        dict(name="qk fwd 1 token", op="qk", back=False, tokens=1, hq=12, hk=12, dim=64, rot=64, dtype="bf16",
             interleaved=False, fused=True),
        # eight sequences of 2048 tokens, width 2048, q and k as views of the fused projection
        dict(name="qk fwd 16384", op="qk", back=False, tokens=16384, hq=16, hk=16, dim=128, rot=128, dtype="bf16",
             interleaved=False, fused=True),
        # its backward pass
        dict(name="qk bwd 16384", op="qk", back=True, tokens=16384, hq=16, hk=16, dim=128, rot=128, dtype="bf16",
             interleaved=False, fused=True),
        # a ragged batch in 32 bits with shared key heads, neighbouring pairs, half of the head rotated
        dict(name="qk bwd f32 ragged", op="qk", back=True, tokens=4099, hq=12, hk=3, dim=64, rot=32, dtype="f32",
             interleaved=True, fused=False),
        # a handful of new tokens: the weights are read once and little is computed
        dict(name="ffn fwd 7 tokens", op="ffn", back=False, tokens=7, d=768, F=2048, act="silu", save=False),
        # eight sequences of 2048 tokens of the 1024-wide model
        dict(name="ffn fwd 16384x1024", op="ffn", back=False, tokens=16384, d=1024, F=2816, act="silu", save=True),
        # a ragged batch of the 768-wide model with the other activation
        dict(name="ffn bwd 4001x768", op="ffn", back=True, tokens=4001, d=768, F=2048, act="gelu", save=True),
        # four sequences of the 2048-wide model: the largest training step
        dict(name="ffn bwd 8192x2048", op="ffn", back=True, tokens=8192, d=2048, F=5632, act="silu", save=True),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "qk", "ffn"])
    if op == "adamw":
        d = log_int(rng, 48, 1024)
        return dict(op=op, tensors=rng.choice(["gains", "rest", "all"]), layers=rng.randint(1, 24), d=d,
                    F=int(d * rng.uniform(2.0, 2.75)), vocab=log_int(rng, 100, 32000), bits=rng.choice([8, 8, 32]),
                    grad=rng.choice(["f32", "bf16"]), copy=rng.random() < 0.3)
    if op == "qk":
        dim = rng.choice([32, 64, 80, 96, 128, 128, 256, 2 * rng.randint(8, 128)])
        hq = rng.randint(1, 24)
        hk = rng.randint(1, hq)
        most = max(1, 16384 * 32 * 128 // ((hq + hk) * dim))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if dtype == "f32":
            most = max(1, most // 2)
        return dict(op=op, back=rng.random() < 0.5, tokens=min(most, log_int(rng, 1, 16384)), hq=hq, hk=hk, dim=dim,
                    rot=rng.choice([dim, dim, dim // 4 * 2]), dtype=dtype, interleaved=rng.random() < 0.3,
                    fused=rng.random() < 0.5)
    back = rng.random() < 0.5
    return dict(op=op, back=back, tokens=log_int(rng, 1, 8192), d=8 * log_int(rng, 8, 256), F=8 * log_int(rng, 16, 704),
                act=rng.choice(["silu", "gelu"]), save=back or rng.random() < 0.5)


def numels(c):
    """Element counts and weight-decay multipliers of a case's tensors."""
    d, hidden = c["d"], [c["d"] * c["d"]] * 4 + [c["d"] * c["F"]] * 3
    gains = [(d, 0.0)] * (2 * c["layers"] + 1)
    if c["tensors"] == "gains":
        return gains
    rest = [(c["vocab"] * d, 1.0)] + gains + [(d * c["vocab"], 1.0)]
    return rest if c["tensors"] == "rest" else rest + [(n, 1.0) for n in hidden] * c["layers"]


def work(c):
    if c["op"] == "adamw":
        n = float(sum(k for k, _ in numels(c)))
        each = 8 + (2 if c["grad"] == "bf16" else 4) + (2 if c["copy"] else 0)
        # 32 bits: both moments read and written.  8 bits: the codes and a scale for 256 of them read and
        # written, and the values that they stand for handed out
        each += 16 if c["bits"] == 32 else 4 + 16 / BLOCK + 8
        return {"bytes": n * each, "flops": 16 * n}
    T = float(c["tokens"])
    if c["op"] == "qk":
        n = T * (c["hq"] + c["hk"]) * c["dim"]
        b = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * b * (3 if c["back"] else 2) + T * (4 * c["rot"] + 8), "flops": n * (16 if c["back"] else 8)}
    d, F = c["d"], c["F"]
    if c["back"]:
        return {"bytes": 2 * (3 * T * d + 3 * T * F + 6 * d * F), "flops": 12 * T * d * F}
    return {"bytes": 2 * (2 * T * d + 3 * d * F + (3 * T * F if c["save"] else 0)), "flops": 6 * T * d * F}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def normal(gen, shape, std, dtype=F32):
    t = torch.empty(shape, dtype=F32, device=DEV).normal_(0.0, std, generator=gen)
    return t if dtype == F32 else t.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"adamw": prepare_adamw, "qk": prepare_qk, "ffn": prepare_ffn}[case["op"]](case, gen)
    s["case"] = case
    if own:
        from paper_2505_23725_b200 import binding
        s["ctx"] = binding.Context(DEV)
        if case["op"] == "adamw":
            s["opt"] = make_adamw(binding, s)
    return s


def prepare_adamw(c, gen):
    tensors = numels(c)
    # every tensor starts on a multiple of 256 elements of flat buffers, as the 8-bit blocks do
    pad = [-(-n // BLOCK) * BLOCK for n, _ in tensors]
    total = sum(pad)
    start = np.concatenate([[0], np.cumsum(pad)[:-1]]).tolist()
    reps = torch.tensor([p // BLOCK for p in pad], device=DEV)
    wd = torch.repeat_interleave(torch.tensor([w for _, w in tensors], dtype=F32, device=DEV), reps)[:, None]
    mask = torch.ones(total, dtype=torch.bool, device=DEV)
    for (n, _), o, p in zip(tensors, start, pad):
        if n < p:
            mask[o + n:o + p] = False
    theta = normal(gen, total, 0.02) * mask
    # the scale of a gradient differs from row to row (token frequencies, layers)
    row = torch.exp(normal(gen, (total // BLOCK, 1), 1.0)) * 1e-3
    grad = ((normal(gen, total, 1.0).view(-1, BLOCK) * row).view(-1) * mask).to(BF16 if c["grad"] == "bf16" else F32)
    s = dict(theta=theta, grad=grad, wd=wd, mask=mask, tensors=tensors, start=start, steps=ADAM_STEPS,
             copy=theta.to(BF16) if c["copy"] else None)
    if c["bits"] == 32:
        s["m"] = (normal(gen, total, 0.3).view(-1, BLOCK) * row).view(-1) * mask
        s["v"] = ((0.5 + torch.rand(total, generator=gen, device=DEV)).view(-1, BLOCK) * row * row).view(-1) * mask
    else:
        s["m"] = (torch.clamp(normal(gen, total, 40.0), -127, 127).round() * mask).to(torch.int8)
        s["v"] = (torch.randint(40, 256, (total,), generator=gen, device=DEV) * mask).to(torch.uint8)
        s["m_scale"] = row.view(-1) / 127
        s["v_scale"] = row.view(-1) * (1.5 / 255)
    return s


def make_adamw(binding, s):
    c = s["case"]

    def views(flat):
        return [flat[o:o + n] for (n, _), o in zip(s["tensors"], s["start"])]

    opt = binding.AdamW(s["ctx"], views(s["theta"]), grads=views(s["grad"]), state_bits=c["bits"],
                        wd_mult=[w for _, w in s["tensors"]], copies=views(s["copy"]) if c["copy"] else None,
                        seed=ADAM_SEED, **ADAM)
    opt.steps = s["steps"]
    opt.state1.copy_(s["m"])
    opt.state2.copy_(s["v"])
    if c["bits"] == 8:
        opt.scale1.copy_(s["m_scale"])
        opt.scale2.copy_(s["v_scale"])
    return opt


def prepare_qk(c, gen):
    T, hq, hk, dim = c["tokens"], c["hq"], c["hk"], c["dim"]
    dtype = BF16 if c["dtype"] == "bf16" else F32

    def heads():
        if c["fused"]:                       # queries, keys and values in one row, as one projection writes them
            qkv = normal(gen, (T, (hq + 2 * hk) * dim), 1.0, dtype)
            return qkv[:, :hq * dim].view(T, hq, dim), qkv[:, hq * dim:(hq + hk) * dim].view(T, hk, dim)
        return normal(gen, (T, hq, dim), 1.0, dtype), normal(gen, (T, hk, dim), 1.0, dtype)

    q, k = heads()
    length = 2048
    inv = 10000.0 ** (-torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64) * 2 / c["rot"])
    ang = torch.arange(length, device=DEV, dtype=torch.float64)[:, None] * inv
    first = int(torch.randint(0, length, (1,), generator=gen, device=DEV))
    s = dict(q=q, k=k, cos=ang.cos().to(F32), sin=ang.sin().to(F32),
             positions=(torch.arange(T, device=DEV) + first) % length,
             gain_q=1.0 + normal(gen, dim, 0.1), gain_k=1.0 + normal(gen, dim, 0.1))
    if c["back"]:
        s["dq"], s["dk"] = normal(gen, (T, hq, dim), 1e-3, dtype), normal(gen, (T, hk, dim), 1e-3, dtype)
    return s


def prepare_ffn(c, gen):
    T, d, F = c["tokens"], c["d"], c["F"]
    s = dict(x=normal(gen, (T, d), 1.0, BF16), w1=normal(gen, (d, F), 0.02, BF16), w3=normal(gen, (d, F), 0.02, BF16),
             w2=normal(gen, (F, d), 0.02, BF16))
    if c["back"]:                            # what the forward pass left, and the gradient of its result
        g, u = s["x"].float() @ s["w1"].float(), s["x"].float() @ s["w3"].float()
        s["saved"] = (g.to(BF16), u.to(BF16), (g * gate(g, c["act"])[0] * u).to(BF16))
        s["dy"] = normal(gen, (T, d), 1e-3, BF16)
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if c["op"] == "adamw":
        return run_adamw(s)
    if c["op"] == "qk":
        how = dict(positions=s["positions"], gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS,
                   interleaved=c["interleaved"])
        if own:
            if c["back"]:
                return s["ctx"].qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["cos"], s["sin"], **how)
            return s["ctx"].qk_norm_rope(s["q"], s["k"], s["cos"], s["sin"], **how)
        cos, sin = s["cos"][s["positions"]][:, None, :], s["sin"][s["positions"]][:, None, :]
        if c["back"]:
            dq, dgq = plain_qk_back(s["dq"], s["q"], s["gain_q"], cos, sin, c["interleaved"])
            dk, dgk = plain_qk_back(s["dk"], s["k"], s["gain_k"], cos, sin, c["interleaved"])
            return dq, dk, dgq, dgk
        return (plain_qk(s["q"], s["gain_q"], cos, sin, c["interleaved"]),
                plain_qk(s["k"], s["gain_k"], cos, sin, c["interleaved"]))
    w1, w3, w2 = s["w1"], s["w3"], s["w2"]
    if own:
        if c["back"]:
            return s["ctx"].gated_ffn_backward(s["dy"], s["x"], w1, w3, w2, s["saved"], activation=c["act"])
        y, saved = s["ctx"].gated_ffn(s["x"], w1, w3, w2, activation=c["act"], save=c["save"])
        return (y,) + saved if c["save"] else y
    if c["back"]:
        return tuple(t.to(BF16) for t in ffn_back(*(t.float() for t in (s["dy"], s["x"], w1, w3, w2) + s["saved"]),
                                                  c["act"]))
    y, g, u, h = ffn(s["x"].float(), w1.float(), w3.float(), w2.float(), c["act"])
    return tuple(t.to(BF16) for t in (y, g, u, h)) if c["save"] else y.to(BF16)


def run_adamw(s):
    c = s["case"]
    if own:
        s["opt"].step()
        # 8-bit codes are handed out as the values that they stand for
        m, v = s["opt"].moments() if c["bits"] == 8 else (s["opt"].state1, s["opt"].state2)
        return [s["theta"], m, v] + ([s["copy"]] if c["copy"] else [])
    s["steps"] += 1
    t, b1, b2 = s["steps"], ADAM["beta1"], ADAM["beta2"]
    g = s["grad"].float().view(-1, BLOCK)
    if c["bits"] == 32:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    else:
        m = s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).square()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    root = v.sqrt()
    theta = s["theta"].view(-1, BLOCK)
    update = (m * f32(1 / (1 - b1 ** t))) / (root * f32(1 / math.sqrt(1 - b2 ** t)) + ADAM["eps"])
    theta = theta - (ADAM["lr"] * update + (ADAM["lr"] * ADAM["weight_decay"]) * s["wd"] * theta)
    s["theta"].copy_(theta.view(-1))
    if c["copy"]:
        s["copy"].copy_(s["theta"])
    if c["bits"] == 32:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return [s["theta"], s["m"], s["v"]] + ([s["copy"]] if c["copy"] else [])
    bits = dither(theta.numel(), t).view(-1, BLOCK)
    (c1, s1), (c2, s2) = encode(m, 127, bits & 0xFFFF), encode(root, 255, bits >> 16)
    c1, c2 = c1.clamp(-127, 127), torch.maximum(c2.clamp(0, 255), (root > 0).float())
    s["m"].copy_(c1.view(-1))
    s["v"].copy_(c2.view(-1))
    s["m_scale"].copy_(s1.view(-1))
    s["v_scale"].copy_(s2.view(-1))
    return [s["theta"], (c1 * s1).view(-1), (c2 * s2).square().view(-1)] + ([s["copy"]] if c["copy"] else [])


def encode(x, top, dither16):
    """Codes floor(x / scale + u) and the scale of each block: its largest magnitude over `top`."""
    a = x.abs().amax(1, keepdim=True)
    inverse = torch.where(a > 1e-36, torch.full_like(a, top) / a, torch.zeros_like(a))
    return (x * inverse + dither16.float() * 2.0 ** -16).floor(), a * f32(1 / top)


def mix(x):
    """A 32-bit integer hash (Mueller): xor-shift and multiply, twice."""
    x = (((x >> 16) ^ x) * 0x45D9F3B) & 0xFFFFFFFF
    x = (((x >> 16) ^ x) * 0x45D9F3B) & 0xFFFFFFFF
    return (x >> 16) ^ x


def dither(n, t):
    """32 random bits for each of n elements at step t: 16 for the first moment's code, 16 for the second's."""
    return mix((torch.arange(n, device=DEV) + mix(mix(ADAM_SEED) + t)) & 0xFFFFFFFF)


def rotate(x, cos, sin, interleaved, sign=1.0):
    """The first 2 * cos.shape[-1] entries of every head turned pair by pair, the others as they are."""
    r = cos.shape[-1]
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if interleaved else (x[..., :r], x[..., r:2 * r])
    y, z = a * cos - sign * b * sin, b * cos + sign * a * sin
    turned = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., 2 * r:]), -1)


def plain_qk(x, gain, cos, sin, interleaved):
    f = x.float()
    n = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    return rotate(n * gain, cos, sin, interleaved).to(x.dtype)


def plain_qk_back(dy, x, gain, cos, sin, interleaved):
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    n = f * r
    dn = rotate(dy.float(), cos, sin, interleaved, -1.0)
    dgain = (dn * n).sum((0, 1))
    e = dn * gain
    return (r * (e - n * (e * n).mean(-1, keepdim=True))).to(x.dtype), dgain


def gate(g, act):
    """sigma and its slope such that act(g) = g sigma: the logistic function of g (silu), or of
    2 sqrt(2 / pi) (g + 0.044715 g^3) (the tanh form of gelu)."""
    if act == "silu":
        p, slope = g, 1.0
    else:
        k = 2.0 * math.sqrt(2.0 / math.pi)
        p, slope = k * (g + 0.044715 * g * g * g), k * (1.0 + 3.0 * 0.044715 * g * g)
    sig = 1.0 / (1.0 + torch.exp(-p))
    return sig, sig * (1.0 - sig) * slope


def ffn(x, w1, w3, w2, act):
    g, u = x @ w1, x @ w3
    h = g * gate(g, act)[0] * u
    return h @ w2, g, u, h


def ffn_back(dy, x, w1, w3, w2, g, u, h, act):
    dh = dy @ w2.T
    sig, dsig = gate(g, act)
    dg, du = dh * u * (sig + g * dsig), dh * (g * sig)
    return dg @ w1.T + du @ w3.T, x.T @ dg, x.T @ du, h.T @ dy


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits, written apart from the plain forms
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"adamw": exact_adamw, "qk": exact_qk, "ffn": exact_ffn}[case["op"]](case, s)


def exact_adamw(c, s):
    b1, b2 = ADAM["beta1"], ADAM["beta2"]
    t = s["steps"] + 1
    g = s["grad"].double()
    if c["bits"] == 32:
        m0, v0 = s["m"].double(), s["v"].double()
    else:
        m0 = s["m"].double() * s["m_scale"].double().repeat_interleave(BLOCK)
        v0 = torch.pow(s["v"].double() * s["v_scale"].double().repeat_interleave(BLOCK), 2)
    m = b1 * m0 + (1.0 - b1) * g
    v = b2 * v0 + (1.0 - b2) * torch.pow(g, 2)
    mhat, vhat = m / (1.0 - b1 ** t), v / (1.0 - b2 ** t)
    wd = ADAM["weight_decay"] * s["wd"].double().view(-1).repeat_interleave(BLOCK)
    theta = s["theta"].double()
    theta = theta - ADAM["lr"] * (mhat / (torch.sqrt(vhat) + ADAM["eps"]) + wd * theta)
    keep = c["bits"] == 32                   # 8-bit moments go by the dither: no value in exact arithmetic
    return [theta, m if keep else None, v if keep else None] + ([theta] if c["copy"] else [])


def exact_qk(c, s):
    pos, half = s["positions"], c["rot"] // 2
    turn = torch.complex(s["cos"].double()[pos], s["sin"].double()[pos])[:, None, :]

    def pairs(x):
        x = x[..., :2 * half]
        return torch.complex(x[..., 0::2], x[..., 1::2]) if c["interleaved"] else torch.complex(x[..., :half], x[..., half:])

    def turned(x, by):
        z = pairs(x) * by
        out = x.clone()
        if c["interleaved"]:
            out[..., 0:2 * half:2], out[..., 1:2 * half:2] = z.real, z.imag
        else:
            out[..., :half], out[..., half:2 * half] = z.real, z.imag
        return out

    def forward(x, gain):
        x = x.double()
        return turned(gain.double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["dim"] + EPS), turn)

    def backward(dy, x, gain):
        x, e = x.double(), turned(dy.double(), turn.conj())
        norm = torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["dim"] + EPS)
        ge = gain.double() * e
        dx = ge / norm - x * (ge * x).sum(-1, keepdim=True) / (c["dim"] * norm.pow(3))
        return dx, (e * x / norm).sum(0).sum(0)

    if not c["back"]:
        return forward(s["q"], s["gain_q"]), forward(s["k"], s["gain_k"])
    dq, dgq = backward(s["dq"], s["q"], s["gain_q"])
    dk, dgk = backward(s["dk"], s["k"], s["gain_k"])
    return dq, dk, dgq, dgk


def exact_ffn(c, s):
    x, w1, w3, w2 = (s[k].double() for k in ("x", "w1", "w3", "w2"))
    k = math.sqrt(2.0 / math.pi)

    def act(g):
        if c["act"] == "silu":
            return g / (1.0 + torch.exp(-g))
        return 0.5 * g * (1.0 + torch.tanh(k * (g + 0.044715 * g ** 3)))

    def slope(g):
        if c["act"] == "silu":
            e = 1.0 / (1.0 + torch.exp(-g))
            return e * (1.0 + g * (1.0 - e))
        th = torch.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th ** 2) * k * (1.0 + 0.134145 * g ** 2)

    if not c["back"]:
        g, u = torch.matmul(x, w1), torch.matmul(x, w3)
        h = act(g) * u
        y = torch.matmul(h, w2)
        return (y, g, u, h) if c["save"] else y
    g, u, h = (t.double() for t in s["saved"])
    dy = s["dy"].double()
    dh = torch.matmul(dy, w2.transpose(0, 1))
    dg, du = dh * u * slope(g), dh * act(g)
    dx = torch.matmul(dg, w1.transpose(0, 1)) + torch.matmul(du, w3.transpose(0, 1))
    return (dx, torch.matmul(x.transpose(0, 1), dg), torch.matmul(x.transpose(0, 1), du),
            torch.matmul(h.transpose(0, 1), dy))
