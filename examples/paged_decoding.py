"""A cache in pages, put together: prompts, continuations that share pages, and attention over few of them.

A small decoder with random weights, grouped heads and rotary positions of three axes (a frame is 2 x 2 tokens: time,
height and width) takes packed prompts, whose rows go into pages, and then decodes one token of each request at a time. Every few
tokens the less likely continuation of each prompt is dropped and the other one forked: the fork shares all pages, and only
the page that both go on writing into is copied.

    python examples/paged_decoding.py [--cache e4m3|bf16] [--requests 4] [--tokens 48] [--picked 0]

`pages_step`, `pages_copy` and `pages_compact` keep the tables; `rotary` turns queries and keys and writes the rows;
`prompt_attention` takes the prompts, `paged_attention` single tokens; `page_bounds` and `page_select` choose the pages that these
attend to.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from draft_decoding import HEAD, Dims, make_weights, rms
from paper_2607_15621_gb300 import fsx

SECTIONS = (16, 24, 24)  # pairs of a head that turn by time, height, width


def places(at: torch.Tensor) -> torch.Tensor:
    """Time, height and width [3, n] of the tokens at these places of their sequences."""
    return torch.stack([at // 4, at // 2 % 2, at % 2])


class PagedDecoder:
    """The model and its pages. Request b's pages are row b of the table; requests come, fork and go by `grow`."""

    def __init__(self, dims: Dims, weights: dict, requests: int, width: int, n_pages: int, page_rows: int = 16, cache: str = "e4m3",
                 picked: int = 0):
        dev, layers = "cuda", range(dims.layers)
        self.dims, self.page_rows, self.picked = dims, page_rows, picked
        self.w = {k: v.to(dev) if isinstance(v, torch.Tensor) else [x.to(dev) for x in v] for k, v in weights.items()}
        rows, hk = n_pages * page_rows, dims.kv_heads
        eight = cache == "e4m3"
        dtype = torch.float8_e4m3fn if eight else torch.bfloat16
        self.k, self.v = ([torch.zeros(rows, hk, HEAD, device=dev, dtype=torch.uint8 if eight else dtype).view(dtype) for _ in layers]
                          for _ in "kv")
        self.ks, self.vs = ([torch.ones(hk, rows, device=dev) if eight else None for _ in layers] for _ in "kv")
        self.bounds = [torch.zeros(n_pages, hk, 2, HEAD, dtype=torch.int8, device=dev) for _ in layers] if picked else []
        self.bound_scale = [torch.ones(hk, n_pages, device=dev) for _ in layers] if picked else []
        self.planes = fsx.page_planes(page_rows, self.k + self.v, self.ks + self.vs if eight else [], self.bounds, self.bound_scale)
        self.width, self.status = width, torch.zeros(1, dtype=torch.int32, device=dev)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        self.table = torch.full((1, width), -1, dtype=torch.int32, device=dev)
        self.lengths = torch.zeros(1, dtype=torch.int64, device=dev)
        self.n_pairs = torch.zeros(1, dtype=torch.int32, device=dev)
        size = fsx.paged_attention_workspace_bytes(requests, dims.heads, hk)
        self.workspace = torch.zeros(size, dtype=torch.uint8, device=dev)  # zeroed once; every call leaves it ready
        self.pairs = fsx.rotary_pairs(SECTIONS)

    def grow(self, source: list[int], new: list[int]) -> torch.Tensor:
        """Request i goes on from request source[i] (-1: from nothing) with new[i] more rows; the new rows' cache rows."""
        B = len(source)
        offsets = torch.tensor([0] + new, device="cuda").cumsum(0)
        table, lengths = torch.empty(B, self.width, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int64, device="cuda")
        rows, pairs = torch.empty(sum(new), dtype=torch.int64, device="cuda"), torch.empty(B, 2, dtype=torch.int32, device="cuda")
        fsx.pages_step(self.table, self.lengths, self.refs, offsets, self.page_rows, table, lengths, self.refs, rows, pairs, self.n_pairs,
                       self.status, source=torch.tensor(source, dtype=torch.int32, device="cuda"))
        fsx.pages_copy(self.planes, pairs, self.n_pairs, self.status)
        self.table, self.lengths = table, lengths
        return rows

    def compact(self):
        """Pages in use to the front of the cache."""
        pairs = torch.empty(len(self.refs) // 2, 2, dtype=torch.int32, device="cuda")
        fsx.pages_compact(self.table, self.lengths, self.refs, self.page_rows, self.table, self.refs, pairs, self.n_pairs, self.status)
        fsx.pages_copy(self.planes, pairs, self.n_pairs, self.status)

    def _forward(self, tokens, at, rows, attend, keys):
        """Logits of packed tokens at these places; their keys and values go to these cache rows."""
        d = self.dims
        x = self.w["emb"][tokens]
        place = places(at)
        for layer in range(d.layers):
            qkv = (rms(x) @ self.w["qkv"][layer]).view(len(tokens), d.heads + 2 * d.kv_heads, HEAD)
            q, k, v = qkv[:, :d.heads], qkv[:, d.heads:d.heads + d.kv_heads], qkv[:, d.heads + d.kv_heads:]
            # in place, columns of the projection's output; single tokens' keys are read from the cache only
            fsx.rotary(q, k, place, self.pairs, self.status, q_out=q, k_out=k if keys else None, v=v, rows=rows, k_cache=self.k[layer],
                       v_cache=self.v[layer], k_scale=self.ks[layer], v_scale=self.vs[layer])
            out = torch.empty(len(tokens), d.heads, HEAD, dtype=q.dtype, device=q.device)
            x = x + attend(layer, q, k, v, out).flatten(1) @ self.w["o"][layer]
        return (rms(x) @ self.w["head"]).float()

    def _bound(self, layer, start):
        fsx.page_bounds(self.k[layer], self.table, self.lengths, self.page_rows, self.bounds[layer], self.bound_scale[layer], self.status,
                        k_scale=self.ks[layer], start=start)

    def prefill(self, prompts: list[list[int]]) -> torch.Tensor:
        """All prompts at once, as new requests; logits of each one's last token."""
        lens = [len(p) for p in prompts]
        rows = self.grow([-1] * len(prompts), lens)
        ends = torch.tensor([0] + lens, device="cuda").cumsum(0)
        at = torch.cat([torch.arange(n, device="cuda") for n in lens])

        def attend(layer, q, k, v, out):
            if self.picked:
                self._bound(layer, None)
            return fsx.prompt_attention(q, k, v, ends, ends, out, self.status)

        logits = self._forward(torch.tensor(sum(prompts, []), device="cuda"), at, rows, attend, True)
        return logits[ends[1:] - 1]

    def step(self, tokens: list[int], source: list[int]) -> torch.Tensor:
        """One more token of each request, which goes on from request source[i]; its logits."""
        rows = self.grow(source, [1] * len(tokens))
        start = self.lengths - 1

        def attend(layer, q, k, v, out):
            chosen = None
            if self.picked:
                self._bound(layer, start)
                chosen = torch.empty(len(tokens), self.dims.kv_heads, self.picked, dtype=torch.int32, device="cuda")
                fsx.page_select(q, self.bounds[layer], self.bound_scale[layer], self.table, self.lengths, self.page_rows, chosen, self.status)
            return fsx.paged_attention(q, self.k[layer], self.v[layer], self.table, self.lengths, self.page_rows, out, self.status,
                                       self.workspace, k_scale=self.ks[layer], v_scale=self.vs[layer], picked=chosen)

        return self._forward(torch.tensor(tokens, device="cuda"), start, rows, attend, False)


def decode(model: PagedDecoder, prompts: list[list[int]], count: int, every: int = 8):
    """Two continuations of `count` tokens of every prompt, the two likeliest tokens first and greedy from there; every `every` tokens
    the less likely one of a prompt gives way to a fork of the other, whose next token is the second likeliest. Returns the sequences and
    the logits that chose each of their tokens."""
    logits = model.prefill(prompts)
    seqs, said, score, source = [], [], [], []
    for b, p in enumerate(prompts):
        for t in logits[b].topk(2).indices.tolist():
            seqs.append(p + [t])
            said.append([logits[b]])
            score.append(float(logits[b].log_softmax(-1)[t]))
            source.append(b)
    for i in range(1, count):
        logits = model.step([s[-1] for s in seqs], source)
        log, best = logits.log_softmax(-1), logits.topk(2).indices.tolist()
        source = list(range(len(seqs)))
        for a in range(0, len(seqs), 2):
            took = [best[a][0], best[a + 1][0]]
            if i % every == 0:
                good = a if score[a] >= score[a + 1] else a + 1
                lost = 2 * a + 1 - good
                seqs[lost], said[lost], score[lost], source[lost] = list(seqs[good]), list(said[good]), score[good], good
                took[good - a], took[lost - a] = best[good]
            for r, t in ((a, took[0]), (a + 1, took[1])):
                seqs[r].append(t)
                said[r].append(logits[source[r]])
                score[r] += float(log[source[r], t])
        if i == count // 2:
            model.compact()
    return seqs, [torch.stack(x) for x in said]


def plain_logits(dims: Dims, weights: dict, tokens: list[int]) -> torch.Tensor:
    """The same model in fp32 without a cache."""
    w = {k: v.float().cuda() if isinstance(v, torch.Tensor) else [x.float().cuda() for x in v] for k, v in weights.items()}
    n, g = len(tokens), dims.heads // dims.kv_heads
    x = w["emb"][torch.tensor(tokens, device="cuda")]
    axis = torch.tensor([a for a, s in enumerate(SECTIONS) for _ in range(s)], device="cuda")
    angle = places(torch.arange(n, device="cuda"))[axis].T.double() * 10000.0 ** (-torch.arange(64, device="cuda").double() / 64)
    c, s = angle.cos().float(), angle.sin().float()

    def turned(y):
        a, b = y[..., :64], y[..., 64:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    hidden = torch.ones(n, n, device="cuda").triu(1).bool()
    for layer in range(dims.layers):
        qkv = (rms(x) @ w["qkv"][layer]).view(n, -1, HEAD).transpose(0, 1)
        q, k, v = qkv[:dims.heads], qkv[dims.heads:dims.heads + dims.kv_heads], qkv[dims.heads + dims.kv_heads:]
        q, k, v = turned(q), turned(k).repeat_interleave(g, 0), v.repeat_interleave(g, 0)
        p = (q @ k.transpose(1, 2) / math.sqrt(HEAD)).masked_fill(hidden, -math.inf).softmax(-1)
        x = x + (p @ v).transpose(0, 1).flatten(1) @ w["o"][layer]
    return rms(x) @ w["head"]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--cache", choices=["e4m3", "bf16"], default="e4m3")
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--picked", type=int, default=0, help="pages that a token attends to; 0: all")
    a = ap.parse_args()
    dims, gen = Dims(), torch.Generator().manual_seed(1)
    weights = make_weights(dims)
    prompts = [torch.randint(dims.vocab, (40 + 23 * b,), generator=gen).tolist() for b in range(a.requests)]
    width = (max(map(len, prompts)) + a.tokens) // 16 + 1
    model = PagedDecoder(dims, weights, 2 * a.requests, width, 2 * a.requests * width, 16, a.cache, a.picked)
    seqs, said = decode(model, prompts, a.tokens)
    used = int((model.refs > 0).sum())
    alone = sum(-(-(len(s) - 1) // 16) for s in seqs)
    print(f"{len(seqs)} continuations of {a.tokens} tokens, {a.cache} pages, status {int(model.status)}")
    print(f"{used} pages in use, {alone} without sharing; the last one is page {int((model.refs > 0).nonzero().max())}")
    want = plain_logits(dims, weights, seqs[0])[len(prompts[0]) - 1:-1]
    print(f"continuation 0: logits {(said[0] - want).abs().max():.3f} from those of the fp32 model without a cache")


if __name__ == "__main__":
    main()
