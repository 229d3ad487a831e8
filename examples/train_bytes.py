"""A small language model on bytes, trained for a few steps: the library's
attention in its layers, its loss over the tied embedding, its gradient clipping
before the optimiser's step; then it continues a text, its keys and values in the
library's paged cache.

    python examples/train_bytes.py [--steps 40] [--layers 2] [--dim 128] [--generate 0]

The text is this repository's own README; everything runs on one GPU in bf16
with fp32 master weights.  Prints the loss (nats per byte) and the gradient's
norm as training goes on, and the bits per byte of a held-out piece at the end.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import paper_2606_28560_gb300 as fa  # noqa: E402

VOCAB, HEAD = 256, 64


class Layer(torch.nn.Module):
    def __init__(self, dim: int):
        super().__init__()
        self.norm1, self.norm2 = torch.nn.RMSNorm(dim), torch.nn.RMSNorm(dim)
        self.qkv = torch.nn.Linear(dim, 3 * dim, bias=False)
        self.out = torch.nn.Linear(dim, dim, bias=False)
        self.up, self.down = torch.nn.Linear(dim, 4 * dim, bias=False), torch.nn.Linear(4 * dim, dim, bias=False)
        self.attention = fa.FibAttention(W=8)

    def forward(self, x, alpha):
        B, T, C = x.shape
        q, k, v = (t.reshape(B, T, C // HEAD, HEAD).transpose(1, 2).contiguous()
                   for t in self.qkv(self.norm1(x)).split(C, dim=-1))
        x = x + self.out(self.attention(q, k, v, alpha=alpha).transpose(1, 2).reshape(B, T, C))
        return x + self.down(torch.nn.functional.silu(self.up(self.norm2(x))))

    def step(self, x, alpha, cache, positions, seqs):
        """The same for new tokens [N, C], whose keys and values go into the cache."""
        N, C = x.shape
        q, k, v = (t.unflatten(1, (C // HEAD, HEAD)) for t in self.qkv(self.norm1(x)).split(C, dim=-1))
        fa.cache_append(cache, k, v, positions, seqs=seqs)
        x = x + self.out(self.attention.cached(q, cache, positions, seqs=seqs, alpha=alpha)[0].reshape(N, C))
        return x + self.down(torch.nn.functional.silu(self.up(self.norm2(x))))


class Model(torch.nn.Module):
    def __init__(self, layers: int, dim: int):
        super().__init__()
        self.embedding = torch.nn.Parameter(torch.randn(VOCAB, dim) * 0.02)
        self.layers = torch.nn.ModuleList(Layer(dim) for _ in range(layers))
        self.norm = torch.nn.RMSNorm(dim)

    def alphas(self):
        thetas = torch.stack([layer.attention.theta.detach() for layer in self.layers]).tolist()
        return [float(a) for a in fa.alpha_schedule("learned", len(self.layers), theta=thetas)]

    def states(self, tokens):
        x = torch.nn.functional.embedding(tokens, self.embedding)
        for layer, a in zip(self.layers, self.alphas()):
            x = layer(x, a)
        return self.norm(x.float())

    def caches(self, length, B, dtype, rows=16):
        """A cache per layer for B sequences of ``length`` tokens, pages of ``rows``."""
        pages = -(-length // rows)
        table = torch.randperm(B * pages).int().view(B, pages).cuda()
        heads = self.embedding.shape[1] // HEAD
        return [fa.PagedCache.empty(B * pages, rows, heads, table, dtype=dtype) for _ in self.layers]

    def steps(self, tokens, caches, positions, seqs, alphas):
        """The states of new tokens [N], one of a sequence or many."""
        x = torch.nn.functional.embedding(tokens, self.embedding)
        for layer, a, cache in zip(self.layers, alphas, caches):
            x = layer.step(x, a, cache, positions, seqs)
        return self.norm(x.float())

    @torch.no_grad()
    def generate(self, prompts, n):
        """The n likeliest bytes after each of the prompts [B, T], one after another."""
        B, T = prompts.shape
        if n < 1:
            return prompts.new_empty(B, 0)
        caches, alphas = self.caches(T + n, B, torch.bfloat16), self.alphas()
        out, tokens = [], prompts.reshape(-1)
        seqs = torch.arange(B, dtype=torch.int32, device="cuda")
        positions = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B)
        with torch.autocast("cuda", dtype=torch.bfloat16):
            x = self.steps(tokens, caches, positions, seqs.repeat_interleave(T), alphas).view(B, T, -1)[:, -1]
            for i in range(n):
                out.append((x @ self.embedding.t()).argmax(-1))
                if i < n - 1:
                    x = self.steps(out[-1], caches, torch.full_like(seqs, T + i), seqs, alphas)
        return torch.stack(out, 1)

    def forward(self, tokens, targets):
        """The mean loss of predicting ``targets`` (-100: no target)."""
        with torch.autocast("cuda", dtype=torch.bfloat16):
            x = self.states(tokens)
        x = x.bfloat16()
        return fa.linear_cross_entropy(x, self.embedding.bfloat16(), targets)


def batch(data, B, T, generator):
    at = torch.randint(0, len(data) - T - 1, (B,), generator=generator)
    rows = torch.stack([data[i:i + T + 1] for i in at.tolist()]).cuda()
    return rows[:, :-1].contiguous(), rows[:, 1:].contiguous()


def train(steps: int = 40, layers: int = 2, dim: int = 128, B: int = 8, T: int = 256, clip: float = 1.0, lr: float = 3e-3,
          seed: int = 0, log=print, generate: int = 0):
    """Returns the losses, the gradient norms and the held-out bits per byte."""
    with open(os.path.join(ROOT, "README.md"), "rb") as f:
        data = torch.tensor(list(f.read()), dtype=torch.int64)
    split = len(data) - max(T + 1, len(data) // 8)
    torch.manual_seed(seed)
    g = torch.Generator().manual_seed(seed)
    model = Model(layers, dim).cuda()
    opt = torch.optim.AdamW(model.parameters(), lr=lr, betas=(0.9, 0.95), weight_decay=0.1)
    losses, norms = [], []
    for step in range(steps):
        loss = model(*batch(data[:split], B, T, g))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        norm = fa.clip_grad_norm_(model.parameters(), clip)
        opt.step()
        losses.append(loss.detach())
        norms.append(norm)
        if log and (step % 10 == 0 or step == steps - 1):
            log(f"step {step:4d}  loss {float(loss):.4f}  gradient norm {float(norm):.3f}")
    with torch.no_grad():
        held = data[split:split + T + 1].cuda()[None]
        bits = float(model(held[:, :-1].contiguous(), held[:, 1:].contiguous())) / math.log(2.0)
    if log:
        log(f"held out: {bits:.3f} bits per byte")
    if log and generate > 0:
        prompt = data[split:split + 64].cuda()[None]
        text = model.generate(prompt, generate)[0].tolist()
        log(repr(bytes(prompt[0].tolist()).decode(errors="replace")) + " -> " + repr(bytes(text).decode(errors="replace")))
    fa.check_status()
    return [float(x) for x in losses], [float(n) for n in norms], bits


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--generate", type=int, default=0, help="bytes to continue a text by")
    a = ap.parse_args()
    train(a.steps, a.layers, a.dim, generate=a.generate)
