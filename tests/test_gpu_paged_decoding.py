"""The operators over a cache in pages together, as the paged decoding example uses them."""
from __future__ import annotations

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paged_decoding as ex

pytestmark = pytest.mark.gpu

# How far logits may lie from the fp32 model's. They have a deviation of 1. 16 bits: some 16 roundings of 2^-9 / sqrt(3) each make
# 0.45 %, 8 deviations 0.04. 8 bits: keys and values are off by 3.6 %, two layers of attention at most as large as the residual
# by 7 %, 8 deviations 0.56.
MARGIN = {"bf16": 0.1, "e4m3": 0.8}


def make(cache, picked, prompts, count, page_rows=16):
    dims = ex.Dims()
    width = (max(map(len, prompts)) + count) // page_rows + 1
    return dims, ex.PagedDecoder(dims, ex.make_weights(dims), 2 * len(prompts), width, 2 * len(prompts) * width, page_rows, cache, picked)


def some_prompts():
    gen = torch.Generator().manual_seed(1)
    return [torch.randint(256, (n,), generator=gen).tolist() for n in (1, 64, 129, 300)]


@pytest.mark.parametrize("page_rows,cache", [(16, "bf16"), (16, "e4m3"), (64, "e4m3")])
def test_continuations_share_pages_and_keep_the_models_logits(page_rows, cache):
    prompts, count = some_prompts(), 30
    dims, model = make(cache, 0, prompts, count, page_rows)
    seqs, said = ex.decode(model, prompts, count, every=7)
    assert int(model.status) == 0 and len(seqs) == 8
    for i, (s, logits) in enumerate(zip(seqs, said)):
        p = prompts[i // 2]
        assert s[:len(p)] == p and len(s) == len(p) + count
        want = ex.plain_logits(dims, ex.make_weights(dims), s)[len(p) - 1:-1]
        assert float((logits - want).abs().max()) <= MARGIN[cache]
    held = torch.zeros_like(model.refs)
    for row, n in zip(model.table, model.lengths.tolist()):
        held.index_add_(0, row[:-(-n // page_rows)].long(), torch.ones(-(-n // page_rows), dtype=torch.int32, device="cuda"))
    assert torch.equal(held, model.refs)
    assert int((model.refs > 1).sum()) > 0  # shared
    model.grow([-1], [0])
    assert int(model.refs.sum()) == 0  # all of them gone


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_a_selection_of_all_pages_is_all_pages_and_of_few_stays_near(cache):
    prompts, count = some_prompts(), 12
    dims, model = make(cache, 0, prompts, count)
    seqs, said = ex.decode(model, prompts, count)
    _, every = make(cache, 24, prompts, count)  # 20 pages and less each
    seqs_every, said_every = ex.decode(every, prompts, count)
    assert int(every.status) == 0
    assert seqs_every == seqs and all(torch.equal(a, b) for a, b in zip(said, said_every))
    _, few = make(cache, 4, prompts, count)
    seqs_few, said_few = ex.decode(few, prompts, count)
    assert int(few.status) == 0 and all(x.isfinite().all() for x in said_few)
    for a, b in zip(said, said_few):
        assert torch.equal(a[0], b[0])  # the first tokens come from the prompts' attention, which sees everything
