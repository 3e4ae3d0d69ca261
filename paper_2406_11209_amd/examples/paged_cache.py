"""An attention layer that is served from a paged compressed cache: two prompts are taken in, one of them is continued in two
ways (a fork, whose shared page is copied when it is written), tokens are added one at a time, a sequence ends and the
pool is brought together.  Every output is set against the same layer on uncompressed keys and values.

    python -m paper_2406_11209_amd.examples.paged_cache [--tokens 2000] [--steps 32]

Needs a GPU.  Inputs are random, projections are random weights: what the layer says means nothing, how far the compressed cache
moves it does.
"""
from __future__ import annotations

import argparse
import math

import torch

from paper_2406_11209_amd.cache import PagedCache

HEADS, GROUPS, DIM, WIDTH = 8, 4, 128, 1024


class Layer:
    """q, k, v of token vectors; keys and values of every sequence kept twice, compressed in pages and as they are."""

    def __init__(self, n_pages: int, page_size: int = 64, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        columns = (HEADS * GROUPS + 2 * HEADS) * DIM
        self.weight = torch.randn(WIDTH, columns, generator=g, device="cuda", dtype=torch.float32) / math.sqrt(WIDTH)
        self.weight = self.weight.to(torch.bfloat16)
        self.cache = PagedCache(DIM, HEADS, n_pages, page_size, work_type="f16")
        self.plain = {}

    def open(self) -> int:
        seq = self.cache.open()
        nothing = torch.empty(0, HEADS, DIM, device="cuda", dtype=torch.bfloat16)
        self.plain[seq] = (nothing, nothing)
        return seq

    def fork(self, seq: int) -> int:
        child = self.cache.fork(seq)
        self.plain[child] = self.plain[seq]
        return child

    def close(self, seq: int) -> None:
        self.cache.close(seq)
        del self.plain[seq]

    def __call__(self, sequences, tokens):
        """tokens[b]: [new, WIDTH] of sequence b -> outputs [all new, HEADS * GROUPS, DIM] and their distance from the
        uncompressed layer's, relative to those."""
        counts = [t.shape[0] for t in tokens]
        qkv = (torch.cat(tokens) @ self.weight).view(sum(counts), -1, DIM)
        q, k, v = qkv.split([HEADS * GROUPS, HEADS, HEADS], dim=1)        # views: the kernels take the strides
        self.cache.extend_and_append(sequences, counts, k, v)
        out = self.cache.attend_sequences(sequences, counts, q)
        want = torch.empty_like(out, dtype=torch.float32)
        first = 0
        for seq, n in zip(sequences, counts):
            keys, values = (torch.cat([old, new[first:first + n]]) for old, new in zip(self.plain[seq], (k, v)))
            self.plain[seq] = (keys, values)
            want[first:first + n] = attention(q[first:first + n].float(), keys.float(), values.float())
            first += n
        return out, float((out.float() - want).norm() / want.norm())


def attention(q, k, v):
    """Causal attention of the last tokens of a sequence, in 32 bits."""
    n, length = q.shape[0], k.shape[0]
    hidden = torch.arange(length, device=q.device)[None, :] > torch.arange(length - n, length, device=q.device)[:, None]
    out = torch.empty_like(q)
    for g in range(q.shape[1]):
        s = q[:, g] @ k[:, g // GROUPS].t() / math.sqrt(DIM)
        out[:, g] = torch.softmax(s.masked_fill(hidden, -math.inf), dim=-1) @ v[:, g // GROUPS]
    return out


def main(tokens: int = 2000, steps: int = 32) -> float:
    """Runs the scene above; returns the largest relative distance met."""
    page = 64
    layer = Layer(n_pages=4 * (-(-(tokens + steps) // page) + 1), page_size=page)
    new = lambda n: torch.randn(n, WIDTH, device="cuda", dtype=torch.bfloat16)
    worst = 0.0

    def report(what, distance):
        nonlocal worst
        worst = max(worst, distance)
        print(f"{what:42s} off by {distance:.4f} of its norm, {layer.cache.pages.free_count} pages free", flush=True)

    a, b = layer.open(), layer.open()
    report(f"prompts of {tokens} and {tokens // 3}", layer([a, b], [new(tokens), new(tokens // 3)])[1])
    c = layer.fork(a)
    report("the first one continued in two ways", layer([a, c], [new(5), new(9)])[1])
    for _ in range(steps):
        distance = layer([a, b, c], [new(1) for _ in range(3)])[1]
    report(f"{steps} steps of one token each", distance)
    layer.close(b)
    moved = layer.cache.compact()
    report(f"one closed, {moved} pages moved", layer([a, c], [new(1), new(1)])[1])
    held = sum(p.numel() * p.element_size() for p in layer.cache.pools)
    full = 2 * layer.cache.n_pages * page * HEADS * DIM * 2
    print(f"pool {held / 2 ** 20:.1f} MiB, {full / 2 ** 20:.1f} MiB as bfloat16")
    return worst


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--tokens", type=int, default=2000)
    parser.add_argument("--steps", type=int, default=32)
    args = parser.parse_args()
    main(args.tokens, args.steps)
