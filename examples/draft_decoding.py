"""Prompts, an 8-bit cache and drafted tokens, put together: greedy decoding of a few requests.

A small decoder with random weights and grouped heads takes packed prompts, writes their keys
and values into one cache per layer, then decodes with drafts: each step sends a tree of guessed tokens through the
model in one pass, keeps the branch that the model itself would have taken and adds its rows to the cache.

    python examples/draft_decoding.py [--cache e4m3|bf16] [--requests 4] [--tokens 48]

`prompt_attention` fills, `cache_write` stores, `tree_attention` decodes, `cache_read` gives rows back.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_15621_gb300 import fsx

HEAD = 128


@dataclass
class Dims:
    layers: int = 2
    heads: int = 8
    kv_heads: int = 2
    width: int = 512
    vocab: int = 256


def make_weights(dims: Dims, seed: int = 0) -> dict:
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s, scale: (torch.randn(*s, generator=gen) * scale).to(torch.bfloat16)
    qkv = (dims.heads + 2 * dims.kv_heads) * HEAD
    return {"emb": normal(dims.vocab, dims.width, scale=1.0), "head": normal(dims.width, dims.vocab, scale=dims.width ** -0.5),
            "qkv": [normal(dims.width, qkv, scale=dims.width ** -0.5) for _ in range(dims.layers)],
            "o": [normal(dims.heads * HEAD, dims.width, scale=(dims.heads * HEAD) ** -0.5) for _ in range(dims.layers)]}


def positions(at: torch.Tensor, width: int) -> torch.Tensor:
    rate = torch.exp(torch.arange(0, width, 2, device=at.device) * (-math.log(1e4) / width))
    angle = at[:, None].float() * rate
    return torch.cat([angle.sin(), angle.cos()], 1)


def rms(x: torch.Tensor) -> torch.Tensor:
    return x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)


class Decoder:
    """The model and its caches; request b owns cache rows [b * room, (b + 1) * room)."""

    def __init__(self, dims: Dims, weights: dict, requests: int, room: int, most_new: int, cache: str = "e4m3"):
        dev = "cuda"
        self.dims, self.room, self.eight = dims, room, cache == "e4m3"
        self.w = {k: v.to(dev) if isinstance(v, torch.Tensor) else [x.to(dev) for x in v] for k, v in weights.items()}
        rows = requests * room
        self.k, self.v = ([torch.zeros(rows, dims.kv_heads, HEAD, device=dev, dtype=torch.uint8 if self.eight else torch.bfloat16)
                           for _ in range(dims.layers)] for _ in "kv")
        if self.eight:
            self.k, self.v = ([x.view(torch.float8_e4m3fn) for x in c] for c in (self.k, self.v))
        self.ks, self.vs = ([torch.ones(dims.kv_heads, rows, device=dev) for _ in range(dims.layers)] for _ in "kv")
        self.starts = torch.arange(requests, device=dev) * room
        self.lengths = [0] * requests  # committed rows
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        size = fsx.tree_attention_workspace_bytes(requests, requests * most_new, dims.heads, dims.kv_heads)
        self.workspace = torch.zeros(size, dtype=torch.uint8, device=dev)  # zeroed once; every call leaves it ready

    def _forward(self, tokens, at, attend):
        """Logits of packed tokens and, per layer, their keys and values (columns of one projection's output)."""
        d, rows = self.dims, []
        x = self.w["emb"][tokens] + positions(at, d.width).to(torch.bfloat16)
        for layer in range(d.layers):
            qkv = (rms(x) @ self.w["qkv"][layer]).view(len(tokens), d.heads + 2 * d.kv_heads, HEAD)
            q, k, v = qkv[:, :d.heads], qkv[:, d.heads:d.heads + d.kv_heads], qkv[:, d.heads + d.kv_heads:]
            x = x + attend(layer, q, k, v, torch.empty(q.shape, dtype=q.dtype, device=q.device)).flatten(1) @ self.w["o"][layer]
            rows.append((k, v))
        return (rms(x) @ self.w["head"]).float(), rows

    def _write(self, layer, k, v, rows):
        if self.eight:
            fsx.cache_write(k, v, rows, self.k[layer], self.v[layer], self.ks[layer], self.vs[layer], self.status)
        else:
            self.k[layer][rows], self.v[layer][rows] = k, v

    def prefill(self, prompts: list[list[int]]) -> torch.Tensor:
        """All prompts at once, one behind another; logits of each one's last token."""
        lens = [len(p) for p in prompts]
        ends = torch.tensor([0] + lens, device="cuda").cumsum(0)
        at = torch.cat([torch.arange(n, device="cuda") for n in lens])
        rows = torch.cat([self.starts[b] + torch.arange(n, device="cuda") for b, n in enumerate(lens)])

        def attend(layer, q, k, v, out):
            return fsx.prompt_attention(q, k, v, ends, ends, out, self.status)

        logits, kv = self._forward(torch.tensor(sum(prompts, []), device="cuda"), at, attend)
        for layer, (k, v) in enumerate(kv):
            self._write(layer, k, v, rows)
        self.lengths = lens
        return logits[ends[1:] - 1]

    def step(self, trees: list[list[tuple[int, int]]]):
        """One pass over a tree of tokens per request, [(token, parent in the tree or -1), ...], parents first.
        Logits of every token, and `keep(paths)`, which commits the tree positions that turned out right."""
        masks, depths = [], []
        for tree in trees:
            m, z = [], []
            for i, (_, parent) in enumerate(tree):
                m.append((m[parent] if parent >= 0 else 0) | 1 << i)  # itself and its ancestors
                z.append(z[parent] + 1 if parent >= 0 else 0)
            masks += m
            depths.append(z)
        first = [0]
        for tree in trees:
            first.append(first[-1] + len(tree))
        new = torch.tensor(first, device="cuda")
        mask = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], device="cuda")
        offsets = torch.tensor([0] + self.lengths, device="cuda").cumsum(0)
        at = torch.tensor([n + z for n, zs in zip(self.lengths, depths) for z in zs], device="cuda")

        def attend(layer, q, k, v, out):
            return fsx.tree_attention(q, k, v, new, mask, self.k[layer], self.v[layer], offsets, out, self.status,
                                      self.workspace, k_scale=self.ks[layer] if self.eight else None,
                                      v_scale=self.vs[layer] if self.eight else None, starts=self.starts)

        logits, kv = self._forward(torch.tensor([t for tree in trees for t, _ in tree], device="cuda"), at, attend)

        def keep(paths):
            took = torch.tensor([first[b] + i for b, path in enumerate(paths) for i in path], device="cuda")
            to = torch.tensor([b * self.room + self.lengths[b] + j for b, path in enumerate(paths) for j in range(len(path))],
                              device="cuda")
            for layer, (k, v) in enumerate(kv):
                self._write(layer, k[took], v[took], to)
            self.lengths = [n + len(path) for n, path in zip(self.lengths, paths)]

        return [logits[first[b]:first[b + 1]] for b in range(len(trees))], keep

    def history(self, layer: int, request: int):
        """A request's committed keys and values in fp32."""
        rows = int(self.starts[request]) + torch.arange(self.lengths[request], device="cuda")
        if not self.eight:
            return self.k[layer][rows].float(), self.v[layer][rows].float()
        k, v = (torch.empty(len(rows), self.dims.kv_heads, HEAD, device="cuda") for _ in "kv")
        return fsx.cache_read(self.k[layer], self.v[layer], self.ks[layer], self.vs[layer], rows, k, v, self.status)


def guess(tokens: list[int], most: int) -> list[tuple[int, int]]:
    """A tree below the last token: what followed its earlier occurrences, two branches at most, by looking back."""
    tree = [(tokens[-1], -1)]
    for start in [i + 1 for i in range(len(tokens) - 2, -1, -1) if tokens[i] == tokens[-1]][:2]:
        parent = 0
        for t in tokens[start:start + (most - 1) // 2]:
            same = [i for i, (u, p) in enumerate(tree) if u == t and p == parent]
            if not same:
                tree.append((t, parent))
            parent = same[0] if same else len(tree) - 1
    return tree[:most]


def decode(model: Decoder, prompts: list[list[int]], count: int, most: int = 8, guess=guess):
    """`count` greedy tokens or a few more behind every prompt; the sequences and the passes that it took. A request that
    has enough sends no tokens."""
    logits = model.prefill(prompts)
    seqs = [p + [int(t)] for p, t in zip(prompts, logits.argmax(-1).tolist())]
    passes = 1
    while min(len(s) - len(p) for s, p in zip(seqs, prompts)) < count:
        trees = [guess(s, most) if len(s) - len(p) < count else [] for s, p in zip(seqs, prompts)]
        logits, keep = model.step(trees)
        paths = []
        for s, tree, lg in zip(seqs, trees, logits):
            best, path = lg.argmax(-1).tolist(), [0] if tree else []
            while tree:  # down the branch that the model takes
                s.append(best[path[-1]])
                nxt = [i for i, (t, p) in enumerate(tree) if p == path[-1] and t == s[-1]]
                if not nxt:
                    break
                path.append(nxt[0])
            paths.append(path)
        keep(paths)
        passes += 1
    return seqs, passes


def plain_logits(dims: Dims, weights: dict, tokens: list[int]) -> torch.Tensor:
    """The same model in fp32 without a cache."""
    w = {k: v.float().cuda() if isinstance(v, torch.Tensor) else [x.float().cuda() for x in v] for k, v in weights.items()}
    n, g = len(tokens), dims.heads // dims.kv_heads
    x = w["emb"][torch.tensor(tokens, device="cuda")] + positions(torch.arange(n, device="cuda"), dims.width)
    hidden = torch.ones(n, n, device="cuda").triu(1).bool()
    for layer in range(dims.layers):
        qkv = (rms(x) @ w["qkv"][layer]).view(n, -1, HEAD).transpose(0, 1)
        q, k, v = qkv[:dims.heads], qkv[dims.heads:dims.heads + dims.kv_heads], qkv[dims.heads + dims.kv_heads:]
        k, v = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
        s = (q @ k.transpose(1, 2) / math.sqrt(HEAD)).masked_fill(hidden, -math.inf).softmax(-1)
        x = x + (s @ v).transpose(0, 1).flatten(1) @ w["o"][layer]
    return rms(x) @ w["head"]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--cache", choices=["e4m3", "bf16"], default="e4m3")
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=48)
    a = ap.parse_args()
    dims, gen = Dims(), torch.Generator().manual_seed(1)
    weights = make_weights(dims)
    prompts = [torch.randint(dims.vocab, (40 + 23 * b,), generator=gen).tolist() for b in range(a.requests)]
    room = max(map(len, prompts)) + a.tokens + 16
    model = Decoder(dims, weights, a.requests, room, 8, a.cache)
    seqs, passes = decode(model, prompts, a.tokens)
    made = sum(len(s) - len(p) for s, p in zip(seqs, prompts))
    print(f"{made} tokens of {a.requests} requests in {passes} passes, {a.cache} cache, status {int(model.status)}")
    want = plain_logits(dims, weights, seqs[0])
    same = (want.argmax(-1)[len(prompts[0]) - 1:-1].cpu() == torch.tensor(seqs[0][len(prompts[0]):])).float().mean()
    print(f"request 0: {100 * same:.0f} % of its tokens are those of the fp32 model without a cache")
    k, _ = model.history(0, 0)
    print(f"request 0 has {k.shape[0]} committed rows")


if __name__ == "__main__":
    main()
