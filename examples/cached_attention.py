"""An attention layer trained with compressed contexts, then answering from a quantised cache.

    python examples/cached_attention.py

One layer: a projection to queries, keys and values (QLinear), norm and rotation of the heads (QHeadNorm), attention, a projection back.
It learns to copy a random sequence for a few steps; then two prompts go through it in chunks and a few tokens one at a time, each
over the paged cache, and the outputs are compared with those of the whole sequences without a cache.
"""
from __future__ import annotations

import os
import sys

import torch
import torch.nn as nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2104_14129_amd import layers as L  # noqa: E402
from paper_2104_14129_amd.cache import PagedCache  # noqa: E402


class Attention(nn.Module):
    def __init__(self, width: int, heads: int, kv_heads: int, dim: int):
        super().__init__()
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.project = L.QLinear(width, (heads + 2 * kv_heads) * dim)
        self.norm = L.QHeadNorm(dim)
        self.back = L.QLinear(heads * dim, width)

    def heads_of(self, x, positions, cos, sin):
        """Normed and rotated queries and keys, values: [tokens, heads, dim] each, out of one projection."""
        x = self.project(x).view(len(x), self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = x.split((self.heads, self.kv_heads, self.kv_heads), 1)
        return *self.norm(q, k, positions, cos, sin), v

    def forward(self, x, positions, cos, sin):
        """A whole sequence, causal."""
        q, k, v = self.heads_of(x, positions, cos, sin)
        k, v = (t.repeat_interleave(self.heads // self.kv_heads, 1) for t in (k, v))
        scores = torch.matmul(q.transpose(0, 1).float(), k.permute(1, 2, 0).float().contiguous()) * self.dim ** -0.5
        hidden = torch.ones(scores.shape[-2:], dtype=torch.bool, device=x.device).triu(1)
        p = scores.masked_fill(hidden, float("-inf")).softmax(-1)
        out = torch.matmul(p, v.transpose(0, 1).float().contiguous()).transpose(0, 1)
        return self.back(out.reshape(len(x), -1).to(x.dtype))

    def answer(self, x, positions, cos, sin, cache, slots, table, lengths, query_start, max_query, max_length):
        """New tokens of several sequences, the rest of which lies in the cache."""
        q, k, v = self.heads_of(x, positions, cos, sin)
        cache.write(k, v, slots)
        out = cache.attend(q, table, lengths, query_start, max_query, max_length)
        return self.back(out.reshape(len(x), -1))


def tables(rows: int, dim: int, device):
    angle = torch.arange(rows, device=device)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device=device) / dim)
    return torch.cos(angle), torch.sin(angle)


def main(steps: int = 5, device: str = "cuda:0") -> dict:
    torch.manual_seed(0)
    width, heads, kv_heads, dim = 256, 8, 2, 64
    layer = Attention(width, heads, kv_heads, dim).to(device)
    cos, sin = tables(1024, dim, device)

    # training: contexts of the linear layers and of the head norm at two bits per element
    L.set_optimization_level("L3", bits=2.0)
    optimizer = torch.optim.Adam(layer.parameters(), lr=1e-3)
    x = torch.randn(300, width, device=device)
    positions = torch.arange(len(x), dtype=torch.int32, device=device)
    losses = []
    for _ in range(steps):
        loss = (layer(x, positions, cos, sin) - x).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))

    # answering: two sequences, chunks of the prompts, then single tokens
    page = 16
    prompts, chunk, more = (150, 41), 64, 6
    total = [n + more for n in prompts]
    sequences = [torch.randn(n, width, device=device) for n in total]
    cache = PagedCache(32, page, kv_heads, dim, device=device)
    table = torch.randperm(32, device=device)[:2 * 10].view(2, 10).int()
    outputs, done = [[], []], [0, 0]
    with torch.no_grad():
        while done != total:
            new = [min(chunk, p - d) if d < p else min(1, t - d) for p, d, t in zip(prompts, done, total)]
            sequence = torch.tensor([s for s, n in enumerate(new) for _ in range(n)], device=device)
            position = torch.tensor([d + i for d, n in zip(done, new) for i in range(n)], device=device)
            rows = torch.cat([s[d:d + n] for s, d, n in zip(sequences, done, new)])
            done = [d + n for d, n in zip(done, new)]
            lengths = torch.tensor(done, dtype=torch.int32, device=device)
            start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=device)
            y = layer.answer(rows, position.int(), cos, sin, cache, cache.slots(table, sequence, position), table, lengths, start, max(new), max(done))
            for s, part in enumerate(y.split(new)):
                outputs[s].append(part)
        off = 0.0
        for s, x in enumerate(sequences):
            want = layer(x, torch.arange(len(x), dtype=torch.int32, device=device), cos, sin)
            off = max(off, float((torch.cat(outputs[s]) - want).norm() / want.norm()))
    return {"losses": losses, "off": off, "cache_bytes": cache.nbytes()}


if __name__ == "__main__":
    result = main()
    print(f"loss {result['losses'][0]:.4f} -> {result['losses'][-1]:.4f}; cached outputs differ by {result['off']:.2e} of their size")
