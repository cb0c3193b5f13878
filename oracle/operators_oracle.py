"""CPU oracle of the operators around the optimizer step.  TEST INFRASTRUCTURE ONLY.

Plain numpy restatements of the definitions, in float64 (the 8-bit AdamW codes in float32, whose
roundings are part of their definition).  Nothing in the product path may import it."""
from __future__ import annotations

import numpy as np

BLOCK = 256


# -- AdamW --------------------------------------------------------------------------------------
def adamw(theta, g, m, v, t, lr, beta1, beta2, eps, wd, bias_correction=True):
    """One step in float64; hyper-parameters as the float32 values the library holds."""
    lr, beta1, beta2, eps, wd = (float(np.float32(x)) for x in (lr, beta1, beta2, eps, wd))
    theta, g, m, v = (np.asarray(x, np.float64) for x in (theta, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    c1 = 1 - beta1 ** t if bias_correction else 1.0
    c2 = 1 - beta2 ** t if bias_correction else 1.0
    return theta - lr * ((m / c1) / (np.sqrt(v / c2) + eps) + wd * theta), m, v


def hash32(x):
    x = np.asarray(x, np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    for _ in range(2):
        x = (((x >> np.uint64(16)) ^ x) * np.uint64(0x45D9F3B)) & mask
    return (x >> np.uint64(16)) ^ x


def dither(n, base, seed, t):
    """(u1, u2) of elements base .. base + n - 1 at step t, float32 in [0, 1)."""
    add = hash32((int(hash32(seed)) + t) & 0xFFFFFFFF)
    r = hash32((np.arange(base, base + n, dtype=np.uint64) + add) & np.uint64(0xFFFFFFFF))
    unit = np.float32(2.0 ** -16)
    return (r & np.uint64(0xFFFF)).astype(np.float32) * unit, (r >> np.uint64(16)).astype(np.float32) * unit


def _encode(x, top, u):
    a = np.abs(x).max(axis=1, keepdims=True)
    with np.errstate(divide="ignore", over="ignore"):
        inv = np.where(a > np.float32(1e-36), np.float32(top) / a, np.float32(0))
    return np.floor(x * inv + u), (a * np.float32(1.0 / top))[:, 0]


def adamw8(g, c1, s1, c2, s2, t, base, seed, beta1, beta2):
    """The 8-bit states of one tensor after a step: c1, c2 padded to whole blocks, s1, s2 one scale per
    block; g without padding.  All arithmetic in float32, one rounding per operation.  Returns the new
    (c1, s1, c2, s2) and the float32 (m, sqrt(v)) that the parameter update uses."""
    f = np.float32
    b1, b2 = f(beta1), f(beta2)
    n, pad = g.size, c1.size
    gp = np.zeros(pad, f)
    gp[:n] = g
    there = (np.arange(pad) < n).reshape(-1, BLOCK)
    gp = gp.reshape(-1, BLOCK)
    m = np.where(there, c1.astype(f).reshape(-1, BLOCK), f(0)) * s1[:, None].astype(f)
    r = np.where(there, c2.astype(f).reshape(-1, BLOCK), f(0)) * s2[:, None].astype(f)
    m = m * b1 + gp * (f(1) - b1)
    root = np.sqrt((r * r) * b2 + (gp * gp) * (f(1) - b2))
    u1, u2 = dither(pad, base, seed, t)
    d1, t1 = _encode(m, 127, u1.reshape(-1, BLOCK))
    d2, t2 = _encode(root, 255, u2.reshape(-1, BLOCK))
    d1 = np.clip(d1, -127, 127)
    d2 = np.maximum(np.clip(d2, 0, 255), (root > 0).astype(f))
    return (d1.astype(np.int8).ravel(), t1.astype(f), d2.astype(np.uint8).ravel(), t2.astype(f),
            m.ravel()[:n], root.ravel()[:n])


# -- norm of queries and keys with the rotation --------------------------------------------------
def _pairs(dim, rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, cos, sin, interleaved, sign=1.0):
    """x [tokens, heads, dim]; cos, sin [tokens, rot / 2]."""
    a, b = _pairs(x.shape[-1], 2 * cos.shape[-1], interleaved)
    y = x.copy()
    c, s = cos[:, None, :], sign * sin[:, None, :]
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def qk_norm(x, gain, cos, sin, eps, interleaved):
    x = np.asarray(x, np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    return rotate(n, cos, sin, interleaved)


def qk_norm_backward(dy, x, gain, cos, sin, eps, interleaved):
    """(dx, dgain, sum of the magnitudes that dgain adds up)."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dn = rotate(dy, cos, sin, interleaved, -1.0)
    e = gain * dn
    dx = r * (e - x * r * (e * x * r).mean(-1, keepdims=True))
    terms = dn * x * r
    return dx, terms.sum((0, 1)), np.abs(terms).sum((0, 1))


# -- gated feed-forward block ---------------------------------------------------------------------
def activation(g, act):
    """(act(g), act'(g))."""
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    k, c = np.sqrt(2.0 / np.pi), 0.044715
    th = np.tanh(k * (g + c * g ** 3))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * k * (1.0 + 3.0 * c * g * g)


def gated_ffn(x, w1, w3, w2, act):
    g, u = x @ w1, x @ w3
    h = activation(g, act)[0] * u
    return h @ w2, g, u, h


def gated_ffn_backward(dy, x, w1, w3, w2, g, u, h, act):
    value, slope = activation(g, act)
    dh = dy @ w2.T
    dg, du = dh * u * slope, dh * value
    return dg @ w1.T + du @ w3.T, x.T @ dg, x.T @ du, h.T @ dy, dg, du
