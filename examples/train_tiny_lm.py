"""A small language model trained with MuLoCo, the whole step on the library's kernels:

  forward / backward   norm of queries and keys with the rotation, gated feed-forward block (layers.py); attention, the
                       other products and the loss are plain torch
  inner step           Muon on the hidden matrices, AdamW with 8-bit states on embedding, head and gains
  outer step           every H steps, over K workers that draw their own batches

The text is synthetic: a walk over the vocabulary whose next token follows from the last one by a fixed table three times
out of four, and is any token otherwise.  Run: python examples/train_tiny_lm.py [--rounds 8] (about a minute of a B200's time at most)."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2505_23725_b200 import binding, configs, layers  # noqa: E402


class Model:
    """Decoder blocks in bf16 over one worker's parameters; `names` are those of configs.llama_tensors plus the
    gains of the query and key norms."""

    def __init__(self, owner, tensors, L, d, heads, length):
        self.owner, self.L, self.d, self.heads, self.dim = owner, L, d, heads, d // heads
        self.index = {t.name: i for i, t in enumerate(tensors)}
        ang = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(self.dim // 2, device="cuda", dtype=torch.float64) * 2 / self.dim)
        self.cos, self.sin = ang.cos().float(), ang.sin().float()

    def leaves(self, theta):
        """Working copies that gather gradients: bf16 matrices, float32 gains."""
        return [t.detach().to(torch.float32 if t.shape[0] == 1 else torch.bfloat16).requires_grad_() for t in theta]

    def loss(self, leaves, tokens):
        p = {n: leaves[i] for n, i in self.index.items()}
        B, S = tokens.shape[0], tokens.shape[1] - 1
        pos = torch.arange(S, device="cuda").repeat(B)

        def norm(x, gain):
            f = x.float()
            return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6) * gain).to(torch.bfloat16)

        x = p["embed"][tokens[:, :-1].reshape(-1)]
        causal = torch.ones(S, S, dtype=torch.bool, device="cuda").tril()
        for l in range(self.L):
            n = norm(x, p[f"l{l}.attn_norm"])
            q, k, v = (n @ p[f"l{l}.{w}"] for w in ("wq", "wk", "wv"))
            q, k = layers.qk_norm_rope(self.owner, q.view(B * S, self.heads, self.dim), k.view(B * S, self.heads, self.dim),
                                       self.cos, self.sin, pos, p[f"l{l}.q_norm"].view(-1), p[f"l{l}.k_norm"].view(-1))
            q, k, v = (t.view(B, S, self.heads, self.dim).transpose(1, 2) for t in (q, k, v))
            a = (q @ k.transpose(-1, -2)).float() * self.dim ** -0.5
            a = a.masked_fill(~causal, float("-inf")).softmax(-1).to(torch.bfloat16) @ v
            x = x + a.transpose(1, 2).reshape(B * S, self.d) @ p[f"l{l}.wo"]
            n = norm(x, p[f"l{l}.ffn_norm"])
            x = x + layers.gated_ffn(self.owner, n, p[f"l{l}.w1"], p[f"l{l}.w3"], p[f"l{l}.w2"])
        logits = (norm(x, p["final_norm"]) @ p["head"]).float()
        return torch.nn.functional.cross_entropy(logits, tokens[:, 1:].reshape(-1))


def workload(L, d, F, vocab, heads, K, H):
    tensors = configs.llama_tensors(L, d, F, vocab=vocab, norms=True)
    for l in range(L):
        for n in ("q_norm", "k_norm"):
            tensors.append(configs.Tensor(f"l{l}.{n}", 1, d // heads, configs.ADAMW, 0, wd_mult=0.0, init="ones"))
    return configs.Workload("tiny-lm", K=K, H=H, J=1, tensors=tensors, muon_lr=0.02, muon_beta=0.9, muon_wd=1e-3,
                            outer_lr=0.7, outer_momentum=0.6, adam_lr=1e-2, adam_state_bits=8)


def batch(gen, table, B, S):
    vocab = table.numel()
    out = [torch.randint(0, vocab, (B,), generator=gen, device="cuda")]
    other = torch.randint(0, vocab, (S, B), generator=gen, device="cuda")
    follow = torch.rand(S, B, generator=gen, device="cuda") < 0.75
    for t in range(S):
        out.append(torch.where(follow[t], table[out[-1]], other[t]))
    return torch.stack(out, 1)


def train(rounds=8, K=2, H=10, L=2, d=128, F=352, vocab=128, heads=2, B=16, S=128, seed=0, quiet=False):
    w = workload(L, d, F, vocab, heads, K, H)
    opt = binding.MuLoCo(w, "cuda:0", init_seed=seed)
    model = Model(opt, w.tensors, L, d, heads, S)
    gens = [torch.Generator(device="cuda").manual_seed(seed + 1 + k) for k in range(K)]
    table = torch.randperm(vocab, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    losses = []
    for r in range(rounds):
        total = 0.0
        for _ in range(H):
            for k in range(K):
                leaves = model.leaves(opt.theta_k[k])
                loss = model.loss(leaves, batch(gens[k], table, B, S))
                loss.backward()
                opt.inner_step(k, [p.grad.float() for p in leaves])
                total += loss.detach()
        opt.outer_sync(-1)
        opt.sync_status()
        losses.append(float(total) / (H * K))
        if not quiet:
            print(f"round {r}: mean loss {losses[-1]:.3f}", flush=True)
    opt.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=8)
    train(ap.parse_args().rounds)
