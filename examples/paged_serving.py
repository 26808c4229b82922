"""Serving one mixer layer over a paged cache: prompts in chunks, then tokens one by one.

    python examples/paged_serving.py [--format e4m3] [--sequences 4] [--tokens 16]

Several sequences of different lengths share one cache. A prompt goes in by chunks (each chunk's
keys and values are written, quantised where the cache is 8-bit, and its queries read the cache),
and then all sequences decode together, a token each per step. The layer is one projection to
queries, keys and values (fewer key/value heads than query heads), the free-energy read, and one
projection back, with random weights and synthetic hidden states. At the end each sequence's keys
and values are read back from the cache and its last row is computed again by the contiguous read.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_07160_gb300 import fem  # noqa: E402


class Layer:
    """Projections and temperatures of one layer; d a head's width."""

    def __init__(self, width, q_heads, heads, d, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.q_heads, self.heads, self.d = q_heads, heads, d
        self.w_in = torch.randn(width, (q_heads + 2 * heads) * d, generator=g, device=device).div_(width ** 0.5).bfloat16()
        self.w_out = torch.randn(q_heads * d, width, generator=g, device=device).div_((q_heads * d) ** 0.5).bfloat16()
        # inverse temperatures about softplus(1.8), their value at initialisation
        self.beta = torch.nn.functional.softplus(1.8 + 0.3 * torch.randn(heads, d, generator=g, device=device))

    def project(self, x):
        """Queries [N, q_heads, d] and keys, values [N, heads, d]: views of one product."""
        y = (x @ self.w_in).view(x.shape[0], -1, self.d)
        return y[:, :self.q_heads], y[:, self.q_heads:self.q_heads + self.heads], y[:, self.q_heads + self.heads:]


class Sequences:
    """Block tables and lengths of a batch of sequences, on the device and as the host knows them."""

    def __init__(self, count, most_tokens, cache):
        self.page = cache.page_size
        self.free = list(range(cache.num_pages))
        self.tables = [[] for _ in range(count)]
        self.lens = [0] * count
        self.block_table = torch.full((count, -(-most_tokens // self.page)), -1, dtype=torch.int32, device=cache.device)
        self.ctx = torch.zeros(count, dtype=torch.int32, device=cache.device)

    def append(self, counts):
        """Room for counts[s] more tokens of every sequence; their slots, sequence by sequence."""
        slots = []
        for s, n in enumerate(counts):
            for pos in range(self.lens[s], self.lens[s] + n):
                if pos // self.page == len(self.tables[s]):
                    self.tables[s].append(self.free.pop())
                    self.block_table[s, len(self.tables[s]) - 1] = self.tables[s][-1]
                slots.append(self.tables[s][pos // self.page] * self.page + pos % self.page)
            self.lens[s] += n
        self.ctx.copy_(torch.tensor(self.lens, dtype=torch.int32))
        return torch.tensor(slots, dtype=torch.int64, device=self.ctx.device)


def step(layer, cache, seqs, x, counts):
    """One pass of the layer over counts[s] new tokens of each sequence (x: their states, [sum, width])."""
    q, k, v = layer.project(x)
    fem.fem_cache_write(cache, k, v, seqs.append(counts))
    offsets = torch.tensor([sum(counts[:s]) for s in range(len(counts) + 1)], dtype=torch.int32, device=x.device)
    out, lse = fem.fem_paged_read(q, cache, layer.beta, offsets, seqs.ctx, seqs.block_table, max_q=max(counts))
    return out.flatten(1) @ layer.w_out, q, out, lse


def serve(prompts, tokens, fmt="e4m3", width=512, q_heads=16, heads=4, d=128, page=64, chunk=256, seed=0):
    """Prompts of the given lengths, then `tokens` decode steps. Returns the largest difference between
    the last rows and the contiguous read of what the cache holds, and the sequences' lengths."""
    device = torch.device("cuda")
    layer = Layer(width, q_heads, heads, d, device, seed)
    dtype = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[fmt]
    most = max(prompts) + tokens
    cache = fem.PagedCache.empty(sum(-(-(p + tokens) // page) for p in prompts), heads, d, page, dtype, device)
    seqs = Sequences(len(prompts), most, cache)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    states = [torch.randn(p, width, generator=g, device=device).bfloat16() for p in prompts]
    x = torch.empty(len(prompts), width, dtype=torch.bfloat16, device=device)
    done = [0] * len(prompts)
    while any(n < p for n, p in zip(done, prompts)):  # chunks of all prompts that are not through
        counts = [min(chunk, p - n) for n, p in zip(done, prompts)]
        y, *_ = step(layer, cache, seqs, torch.cat([s[n:n + c] for s, n, c in zip(states, done, counts)]), counts)
        ends = [sum(counts[:s + 1]) - 1 for s in range(len(counts))]
        for s, c in enumerate(counts):
            if c:
                x[s] = y[ends[s]]
        done = [n + c for n, c in zip(done, counts)]
    for _ in range(tokens):
        x, q, out, lse = step(layer, cache, seqs, x, [1] * len(prompts))
    fem.check_device_error()

    # what the cache holds, read back, through the contiguous read
    total = sum(seqs.lens)
    offsets = torch.tensor([sum(seqs.lens[:s]) for s in range(len(prompts) + 1)], dtype=torch.int32, device=device)
    k, v = fem.fem_cache_gather(cache, seqs.block_table, torch.zeros_like(seqs.ctx), offsets, total)
    group, worst = q_heads // heads, 0.0
    for s in range(len(prompts)):
        rows = slice(int(offsets[s]), int(offsets[s + 1]))
        ks, vs = (t[rows].transpose(0, 1).repeat_interleave(group, 0).contiguous()[None] for t in (k, v))
        ref, _ = fem.fem_decode(q[s][None].contiguous(), ks, vs, layer.beta.repeat_interleave(group, 0).contiguous())
        worst = max(worst, (out[s].float() - ref[0]).abs().max().item())
    return worst, seqs.lens


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--format", choices=["bf16", "e4m3"], default="e4m3")
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=16)
    a = ap.parse_args(argv)
    prompts = [100 + 371 * s for s in range(a.sequences)]
    worst, lens = serve(prompts, a.tokens, a.format)
    print(f"{a.sequences} sequences of {lens} positions, {a.format} cache: last rows within {worst:.2e} of the contiguous read")


if __name__ == "__main__":
    main()
