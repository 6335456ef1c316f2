"""Prompt attention, the 8-bit cache and tree attention together, as the decoding example uses them."""
from __future__ import annotations

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import draft_decoding as ex

pytestmark = pytest.mark.gpu

# How far below the fp32 model's best logit a chosen token's may lie. Logits have a deviation of 1. 16 bits: some 14
# roundings of 2^-9 / sqrt(3) each make 0.4 %, 0.6 % of a difference, 8 deviations 0.05. 8 bits: keys and values are off by
# 3.6 %, two layers of attention at most as large as the residual by 7 %, a difference by 10 %.
MARGIN = {"bf16": 0.1, "e4m3": 0.8}


def short_of_best(dims, weights, seq, start):
    logits = ex.plain_logits(dims, weights, seq)[start - 1:-1]
    took = logits.gather(1, torch.tensor(seq[start:], device="cuda")[:, None])[:, 0]
    return float((logits.amax(1) - took).max())


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_decoding_with_and_without_drafts(cache):
    dims, count = ex.Dims(), 20
    weights = ex.make_weights(dims)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(dims.vocab, (n,), generator=gen).tolist() for n in (1, 60, 129, 300)]
    room = 300 + count + 16
    known, passes = ex.decode(ex.Decoder(dims, weights, 4, room, 8, cache), prompts, count, most=1)
    assert passes == count

    def told(seq, most):  # the continuation that is known by now, and a wrong branch at every token
        full = next(k for k in known if k[0] == seq[0])
        tree = [(seq[-1], -1)]
        parent = 0
        for t in full[len(seq):len(seq) + (most - 1) // 2]:
            tree.append(((t + 1) % dims.vocab, parent))
            tree.append((t, parent))
            parent = len(tree) - 1
        return tree

    model = ex.Decoder(dims, weights, 4, room, 8, cache)
    drafted, fewer = ex.decode(model, prompts, count, guess=told)
    assert int(model.status) == 0 and fewer < passes
    for seqs in (known, drafted):
        for p, s in zip(prompts, seqs):
            assert len(s) - len(p) >= count and s[:len(p)] == p
            assert short_of_best(dims, weights, s, len(p)) <= MARGIN[cache]
    k, v = model.history(1, 3)
    assert k.shape == (model.lengths[3], dims.kv_heads, 128) and k.isfinite().all() and v.abs().max() > 0
