"""Measured cases of the operators that complete a decoder's training step: causal attention over packed sequences with
shared key heads, layer norm (centred or not, with the residual sum in front of it) and embedding lookup, each forward
and backward.

`run` computes an operator in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, with
`own` set, through the library.  Sizes are those of the benchmark configurations (widths 768 / 1024 / 2048, heads of 64
and 128, vocabulary 32000, sequences of 2048) and odd ones around them.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
EPS = 2.0 ** -20                             # (a value that 32 bits hold)


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # the first token of a text, 12 heads of 64: latency
        dict(name="attention fwd 1 token", op="attention", back=False, lengths="1", tail=0, hq=12, hk=12, dim=64,
             fused=True, lseed=1),
        # eight sequences of 2048 tokens at width 2048, q, k and v as views of the fused projection
        dict(name="attention fwd 8x2048", op="attention", back=False, lengths="8x2048", tail=0, hq=16, hk=16, dim=128,
             fused=True, lseed=1),
        # its backward pass
        dict(name="attention bwd 8x2048", op="attention", back=True, lengths="8x2048", tail=0, hq=16, hk=16, dim=128,
             fused=True, lseed=1),
        # documents of very different lengths packed into a padded batch, four query heads to a key head
        dict(name="attention bwd packed", op="attention", back=True, lengths="23 of 7900", tail=292, hq=12, hk=3,
             dim=64, fused=False, lseed=7),
        # one long text: the largest
        dict(name="attention fwd 1x16384", op="attention", back=False, lengths="1x16384", tail=0, hq=16, hk=4, dim=128,
             fused=False, lseed=1),
        # one new token at width 768: latency
        dict(name="norm fwd 1 token", op="norm", back=False, tokens=1, d=768, center=False, bias=False, residual=True,
             dtype="bf16"),
        # the norm in front of a feed-forward block, with the sum of the residual stream: eight sequences of 2048
        dict(name="norm fwd 16384x2048", op="norm", back=False, tokens=16384, d=2048, center=False, bias=False,
             residual=True, dtype="bf16"),
        # its backward pass in the 1024-wide model, centred and with a bias; the stream's own gradient joins
        dict(name="norm bwd 16384x1024", op="norm", back=True, tokens=16384, d=1024, center=True, bias=True,
             residual=True, dtype="bf16"),
        # 32 bits, a ragged batch and an odd width
        dict(name="norm bwd f32 ragged", op="norm", back=True, tokens=4099, d=771, center=True, bias=True,
             residual=False, dtype="f32"),
        # the tokens of eight sequences of 2048 looked up in the 1024-wide table, scaled
        dict(name="embedding fwd 16384x1024", op="embedding", back=False, tokens=16384, vocab=32000, d=1024,
             dtype="bf16"),
        # the table's gradient for a ragged batch of the 768-wide model, in 16 bits
        dict(name="embedding bwd 4001x768", op="embedding", back=True, tokens=4001, vocab=32000, d=768, dtype="bf16"),
        # the same in 32 bits for eight sequences of 2048 at width 2048
        dict(name="embedding bwd 16384x2048", op="embedding", back=True, tokens=16384, vocab=32000, d=2048,
             dtype="f32"),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed() if c["op"] == "attention")
    op = rng.choice(["attention", "attention", "norm", "embedding"])
    if op == "attention":
        while True:
            group = rng.choice([1, 1, 2, 3, 4, 8])
            hk = rng.randint(1, max(1, 24 // group))
            total = log_int(rng, 1, 16384)
            n = min(total, log_int(rng, 1, 64))
            c = dict(op=op, back=rng.random() < 0.6, lengths=f"{n} of {total}", tail=rng.choice([0, 0, rng.randint(1, 500)]),
                     hq=group * hk, hk=hk, dim=rng.choice([32, 64, 64, 80, 96, 128, 128, 8 * rng.randint(1, 16)]),
                     fused=rng.random() < 0.5, lseed=rng.randint(1, 10 ** 6))
            if work(c)["flops"] <= most:
                return c
    if op == "norm":
        d = rng.choice([8 * log_int(rng, 8, 512), log_int(rng, 16, 4096)])
        back = rng.random() < 0.6
        dtype = rng.choice(["bf16", "bf16", "f32"])
        limit = 16384 * 2048 // ((2 if back else 1) * (2 if dtype == "f32" else 1))
        center = rng.random() < 0.5
        return dict(op=op, back=back, tokens=max(1, min(log_int(rng, 1, 65536), limit // d)), d=d, center=center,
                    bias=center and rng.random() < 0.7, residual=rng.random() < 0.5, dtype=dtype)
    d = rng.choice([8 * log_int(rng, 6, 256), log_int(rng, 24, 2048)])
    vocab = log_int(rng, 100, 32000)
    return dict(op=op, back=rng.random() < 0.7, tokens=log_int(rng, 1, 16384), vocab=vocab, d=d,
                dtype=rng.choice(["bf16", "f32"]))


def sequence_lengths(c):
    """Lengths of the packed sequences: "n x m" is n of m tokens, "n of m" n of very different lengths, m in all."""
    if "x" in c["lengths"]:
        n, m = c["lengths"].split("x")
        return [int(m)] * int(n)
    if " of " not in c["lengths"]:
        return [int(c["lengths"])]
    n, m = (int(t) for t in c["lengths"].split(" of "))
    state, weights = c["lseed"], []
    for _ in range(n):                       # lengths differ by up to a factor of e^3
        state = (state * 1103515245 + 12345) % 2 ** 31
        weights.append(math.exp(3.0 * state / 2 ** 31))
    out = [1 + int((m - n) * w / sum(weights)) for w in weights]
    out[-1] += m - sum(out)
    return out


def work(c):
    if c["op"] == "attention":
        lengths = sequence_lengths(c)
        tokens = float(sum(lengths) + c["tail"])
        pairs = sum(0.5 * n * (n + 1) for n in lengths)
        q, k = tokens * c["hq"] * c["dim"], tokens * c["hk"] * c["dim"]
        if c["back"]:                        # q, k, v, o, do and lse in, dq, dk, dv out; five products
            return {"bytes": 2 * (4 * q + 4 * k) + 4 * tokens * c["hq"], "flops": 10 * pairs * c["hq"] * c["dim"]}
        return {"bytes": 2 * (2 * q + 2 * k) + 4 * tokens * c["hq"], "flops": 4 * pairs * c["hq"] * c["dim"]}
    b = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        n, extra = float(c["tokens"]) * c["d"], 8 * c["tokens"] + 8 * c["d"]
        if c["back"]:
            return {"bytes": n * b * (4 if c["residual"] else 3) + extra, "flops": 12 * n}
        return {"bytes": n * b * (4 if c["residual"] else 2) + extra, "flops": 8 * n}
    n, table = float(c["tokens"]) * c["d"], float(c["vocab"]) * c["d"]
    if c["back"]:                            # gradients in, every row of the table's gradient out
        return {"bytes": n * 2 + 8 * c["tokens"] + table * b, "flops": n}
    used = min(c["tokens"], c["vocab"]) * float(c["d"])
    return {"bytes": used * b + 8 * c["tokens"] + n * b, "flops": n}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def normal(gen, shape, std, dtype=F32):
    t = torch.empty(shape, dtype=F32, device=DEV).normal_(0.0, std, generator=gen)
    return t if dtype == F32 else t.to(dtype)


def type_of(c):
    return BF16 if c["dtype"] == "bf16" else F32


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"attention": prepare_attention, "norm": prepare_norm, "embedding": prepare_embedding}[case["op"]](case, gen)
    s["case"] = case
    if own:
        from paper_2505_23725_b200 import binding
        s["ctx"] = binding.Context(DEV)
        if case["op"] == "attention":        # made once for a batch: all layers, forward and backward, use it
            s["seq"] = binding.Sequences(s["ctx"], s["lengths"], tokens=s["q"].shape[0])
    return s


def prepare_attention(c, gen):
    lengths, hq, hk, dim = sequence_lengths(c), c["hq"], c["hk"], c["dim"]
    T = sum(lengths) + c["tail"]
    if c["fused"]:                           # queries, keys and values in one row, as one projection writes them
        qkv = normal(gen, (T, hq + 2 * hk, dim), 1.0, BF16)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        q, k, v = (normal(gen, (T, h, dim), 1.0, BF16) for h in (hq, hk, hk))
    s = dict(lengths=lengths, q=q, k=k, v=v, scale=dim ** -0.5)
    if c["back"]:                            # what the forward pass left, and the gradient of its result
        o, lse = plain_attention(q, k, v, lengths, s["scale"])
        s["o"], s["lse"], s["do"] = o, lse, normal(gen, (T, hq, dim), 1e-3, BF16)
    return s


def prepare_norm(c, gen):
    T, d, dtype = c["tokens"], c["d"], type_of(c)
    # entries of a residual stream: a scale per token, a few wide columns, a small common part
    spread = torch.exp(normal(gen, (T, 1), 0.3)) * torch.exp(normal(gen, (d,), 0.5))
    x = (normal(gen, (T, d), 1.0) * spread + 0.2).to(dtype)
    s = dict(x=x, weight=1.0 + normal(gen, d, 0.1), bias=normal(gen, d, 0.1) if c["bias"] else None)
    if c["back"]:
        f = x.float()
        s["mean"] = f.mean(1) if c["center"] else None
        var = f.square().mean(1) if not c["center"] else (f - s["mean"][:, None]).square().mean(1)
        s["rstd"] = torch.rsqrt(var + EPS)
        s["dy"] = normal(gen, (T, d), 1e-3, dtype)
        s["dh"] = normal(gen, (T, d), 1e-3, dtype) if c["residual"] else None
    else:
        s["residual"] = normal(gen, (T, d), 0.5, dtype) if c["residual"] else None
    return s


def prepare_embedding(c, gen):
    T, V, d = c["tokens"], c["vocab"], c["d"]
    # word frequencies: the k-th most frequent token has a share that falls like 1 / k, tokens in no order
    rank = (V + 1.0) ** torch.rand(T, generator=gen, device=DEV, dtype=torch.float64) - 1.0
    names = torch.randperm(V, generator=gen, device=DEV)
    s = dict(ids=names[rank.long().clamp(0, V - 1)], scale=float(math.sqrt(2 ** round(math.log2(d)))))
    if c["back"]:
        s["dout"] = normal(gen, (T, d), 1e-3, BF16)
    else:
        s["table"] = normal(gen, (V, d), 0.02, type_of(c))
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if c["op"] == "attention":
        if own:
            if c["back"]:
                return s["ctx"].causal_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["seq"],
                                                          scale=s["scale"])
            return s["ctx"].causal_attention(s["q"], s["k"], s["v"], s["seq"], scale=s["scale"])
        if c["back"]:
            return plain_attention_back(s["do"], s["q"], s["k"], s["v"], s["lengths"], s["scale"])
        return plain_attention(s["q"], s["k"], s["v"], s["lengths"], s["scale"])
    if c["op"] == "norm":
        if own:
            if c["back"]:
                dx, dw, db = s["ctx"].layer_norm_backward(s["dy"], s["x"], s["rstd"], s["mean"], weight=s["weight"],
                                                          dh=s["dh"], bias=c["bias"])
                return (dx, dw, db) if c["bias"] else (dx, dw)
            y, h, rstd, mean = s["ctx"].layer_norm(s["x"], weight=s["weight"], bias=s["bias"], residual=s["residual"],
                                                   eps=EPS, center=c["center"])
            return [t for t in (y, h if c["residual"] else None, rstd, mean) if t is not None]
        return plain_norm_back(s, c) if c["back"] else plain_norm(s, c)
    if c["back"]:
        if own:
            return s["ctx"].embedding_backward(s["dout"], s["ids"], c["vocab"], scale=s["scale"], dtype=type_of(c))
        out = torch.zeros(c["vocab"], c["d"], dtype=F32, device=DEV)
        return out.index_add_(0, s["ids"], s["dout"].float()).mul_(s["scale"]).to(type_of(c))
    if own:
        return s["ctx"].embedding(s["ids"], s["table"], scale=s["scale"])
    return (s["table"][s["ids"]].float() * s["scale"]).to(type_of(c))


def spans(lengths, heads):
    """(first token, end, first head, end) of the pieces whose scores are held at once: a sequence, and as many of its
    heads as stay below 2^28 scores."""
    at = 0
    for n in lengths:
        step = max(1, min(heads, 2 ** 28 // max(1, n * n)))
        for h in range(0, heads if n else 0, step):
            yield at, at + n, h, min(heads, h + step)
        at += n


def scores(q, k, scale):
    """Scores of one piece, [heads, n, n]: -inf where the key comes after the query."""
    n = q.shape[1]
    later = torch.arange(n, device=DEV)[None, :] > torch.arange(n, device=DEV)[:, None]
    return (q @ k.transpose(1, 2) * scale).masked_fill_(later, float("-inf"))


def piece(t, a, b, heads):
    """The given heads of tokens a .. b in 32 bits, [heads, tokens, dim]."""
    return t[a:b, heads].float().transpose(0, 1)


def plain_attention(q, k, v, lengths, scale):
    T, hq, _ = q.shape
    group = hq // k.shape[1]
    o, lse = torch.zeros(q.shape, dtype=BF16, device=DEV), torch.zeros(hq, T, dtype=F32, device=DEV)
    for a, b, h0, h1 in spans(lengths, hq):
        heads = torch.arange(h0, h1, device=DEV)
        x = scores(piece(q, a, b, heads), piece(k, a, b, heads // group), scale)
        top = x.amax(-1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(-1, keepdim=True)
        o[a:b, h0:h1] = (e @ piece(v, a, b, heads // group) / total).transpose(0, 1).to(BF16)
        lse[h0:h1, a:b] = (top + total.log())[..., 0]
    return o, lse


def plain_attention_back(do, q, k, v, lengths, scale):
    T, hq, dim = q.shape
    hk = k.shape[1]
    group = hq // hk
    dq = torch.zeros(T, hq, dim, dtype=F32, device=DEV)
    dk, dv = (torch.zeros(T, hk, dim, dtype=F32, device=DEV) for _ in range(2))
    for a, b, h0, h1 in spans(lengths, hq):
        heads = torch.arange(h0, h1, device=DEV)
        fq, fk, fv, g = (piece(t, a, b, h) for t, h in ((q, heads), (k, heads // group), (v, heads // group), (do, heads)))
        x = scores(fq, fk, scale)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        dp = g @ fv.transpose(1, 2)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        dq[a:b, h0:h1] = (ds @ fk).transpose(0, 1)
        dk[a:b].index_add_(1, heads // group, (ds.transpose(1, 2) @ fq).transpose(0, 1))
        dv[a:b].index_add_(1, heads // group, (p.transpose(1, 2) @ g).transpose(0, 1))
    return dq.to(BF16), dk.to(BF16), dv.to(BF16)


def plain_norm(s, c):
    f = s["x"].float()
    if c["residual"]:
        f = f + s["residual"].float()
    mean = f.mean(1, keepdim=True) if c["center"] else torch.zeros(1, 1, device=DEV)
    rstd = torch.rsqrt((f - mean).square().mean(1, keepdim=True) + EPS)
    y = (f - mean) * rstd * s["weight"]
    if c["bias"]:
        y = y + s["bias"]
    out = [y.to(type_of(c))] + ([f.to(type_of(c))] if c["residual"] else []) + [rstd[:, 0]]
    return out + ([mean[:, 0]] if c["center"] else [])


def plain_norm_back(s, c):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    n = (s["x"].float() - s["mean"][:, None] if c["center"] else s["x"].float()) * rstd
    e = dy * s["weight"]
    dx = e - n * (e * n).mean(1, keepdim=True)
    if c["center"]:
        dx = dx - e.mean(1, keepdim=True)
    dx = dx * rstd
    if c["residual"]:
        dx = dx + s["dh"].float()
    out = (dx.to(type_of(c)), (dy * n).sum(0))
    return out + (dy.sum(0),) if c["bias"] else out


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
    return {"attention": exact_attention, "norm": exact_norm, "embedding": exact_embedding}[case["op"]](case, s)


def exact_attention(c, s):
    """Head by head: log-sum-exp of the scores, its exponential weights, and for the gradients the derivative of a softmax
    written out as weights times (dp minus do . o)."""
    lengths, scale = s["lengths"], s["scale"]
    q, k, v = s["q"], s["k"], s["v"]
    T, hq, dim = q.shape
    group = hq // k.shape[1]
    o, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(hq, T, dtype=torch.float64, device=DEV)
    dq = torch.zeros_like(o)
    dk, dv = (torch.zeros(k.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    end = 0
    for n in lengths:
        a, end = end, end + n
        allowed = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        for h in range(hq if n else 0):
            qh, kh, vh = q[a:end, h].double(), k[a:end, h // group].double(), v[a:end, h // group].double()
            logits = torch.einsum("id,jd->ij", qh, kh).mul_(scale).masked_fill_(~allowed, -math.inf)
            z = torch.logsumexp(logits, 1)
            w = logits.sub_(z[:, None]).exp_()
            out = torch.einsum("ij,jd->id", w, vh)
            o[a:end, h], lse[h, a:end] = out, z
            if c["back"]:
                g = s["do"][a:end, h].double()
                dv[a:end, h // group] += torch.einsum("ij,id->jd", w, g)
                dlogits = torch.einsum("id,jd->ij", g, vh).sub_(torch.einsum("id,id->i", g, out)[:, None]).mul_(w)
                dq[a:end, h] = torch.einsum("ij,jd->id", dlogits, kh) * scale
                dk[a:end, h // group] += torch.einsum("ij,id->jd", dlogits, qh) * scale
    return (dq, dk, dv) if c["back"] else (o, lse)


def exact_norm(c, s):
    x = s["x"].double()
    if not c["back"] and c["residual"]:
        x = x + s["residual"].double()
    d = c["d"]
    shift = x.sum(1, keepdim=True) / d if c["center"] else torch.zeros(x.shape[0], 1, dtype=torch.float64, device=DEV)
    spread = torch.sqrt((x - shift).pow(2).sum(1, keepdim=True) / d + EPS)
    unit = (x - shift) / spread
    if not c["back"]:
        y = torch.addcmul(s["bias"].double() if c["bias"] else torch.zeros(d, dtype=torch.float64, device=DEV), unit,
                          s["weight"].double())
        out = [y] + ([x] if c["residual"] else []) + [1.0 / spread[:, 0]]
        return out + ([shift[:, 0]] if c["center"] else [])
    dy = s["dy"].double()
    du = dy * s["weight"].double()
    # x -> (x - shift) / spread: the part of du along unit (and, centred, along ones) does not pass
    dx = du - unit * (torch.einsum("td,td->t", du, unit) / d)[:, None]
    if c["center"]:
        dx = dx - du.sum(1, keepdim=True) / d
    dx = dx / spread
    if c["residual"]:
        dx = dx + s["dh"].double()
    out = (dx, torch.einsum("td,td->d", dy, unit))
    return out + (dy.sum(0),) if c["bias"] else out


def exact_embedding(c, s):
    if not c["back"]:
        return torch.index_select(s["table"], 0, s["ids"]).double() * s["scale"]
    order = torch.argsort(s["ids"], stable=True)
    used, counts = torch.unique_consecutive(s["ids"][order], return_counts=True)
    grads = s["dout"].double()[order]
    ends = torch.cumsum(counts, 0)
    out = torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device=DEV)
    which = torch.bucketize(torch.arange(c["tokens"], device=DEV), ends, right=True)
    sums = torch.zeros(used.numel(), c["d"], dtype=torch.float64, device=DEV).index_add_(0, which, grads)
    out[used] = sums * s["scale"]
    return out
