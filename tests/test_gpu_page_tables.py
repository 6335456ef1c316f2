"""fsx_pages_step, fsx_pages_compact and fsx_pages_copy on the GPU against the lists of the oracle."""
from __future__ import annotations

import os
import random
import sys

import pytest
import torch

from oracle import pages_oracle as po
from paper_2607_15621_gb300 import fsx

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_pages_oracle_pins import random_state

pytestmark = pytest.mark.gpu


def ints(v, t=torch.int32):
    return torch.tensor(v, dtype=t, device="cuda")


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def table_of(state, fill=-1):
    return ints([row + [fill] * (state.width - len(row)) for row in state.pages]).view(len(state.pages), state.width)


def offsets(new):
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    return ints(at, torch.int64)


def step(state, source, new, in_place=False, source_given=True):
    B, total = len(new), sum(new)
    table, lengths, refs = table_of(state), ints(state.lengths, torch.int64), ints(state.refs)
    a = dict(table_out=table if in_place else torch.full((B, state.width), 55, dtype=torch.int32, device="cuda"),
             lengths_out=lengths if in_place else torch.full((B,), 55, dtype=torch.int64, device="cuda"),
             refs_out=refs if in_place else torch.full_like(refs, 55), rows=torch.full((total,), 55, dtype=torch.int64, device="cuda"),
             pairs=torch.full((B, 2), 55, dtype=torch.int32, device="cuda"), n_pairs=torch.full((1,), 55, dtype=torch.int32, device="cuda"))
    st = status()
    fsx.pages_step(table, lengths, refs, offsets(new), state.page_rows, status=st, source=ints(source) if source_given else None, **a)
    return a, int(st)


def same(a, want, rows, pairs, in_place=False):
    table = a["table_out"].cpu().tolist()
    for got, row in zip(table, want.pages):
        assert got[:len(row)] == row
        assert in_place or all(x == -1 for x in got[len(row):])
    assert a["lengths_out"].tolist() == want.lengths and a["refs_out"].tolist() == want.refs
    assert a["rows"].tolist() == rows
    n = int(a["n_pairs"])
    assert [tuple(p) for p in a["pairs"][:n].tolist()] == pairs and (a["pairs"][n:] == 55).all()


@pytest.mark.parametrize("seed", range(30))
def test_steps_of_random_states(seed):
    rng = random.Random(seed)
    page_rows = rng.choice([16, 16, 32, 256])
    state = random_state(rng, rng.randint(1, 40), rng.randint(10, 200), rng.randint(2, 9), page_rows)
    for _ in range(3):
        B = rng.randint(1, 40)
        source = [rng.randrange(-1, len(state.pages)) for _ in range(B)]
        new = [rng.choice([0, 1, 1, 2, page_rows, 3 * page_rows]) for _ in source]
        a, st = step(state, source, new)
        refused = any((state.lengths[s] if s >= 0 else 0) + n > state.width * page_rows for s, n in zip(source, new))
        state, rows, pairs, short = state.step(source, new)
        same(a, state, rows, pairs)
        assert st in ((fsx.FSX_ERR_DEVICE_ARG, 3) if refused and short else (fsx.FSX_ERR_DEVICE_ARG,) if refused else (3,) if short else (0,))


@pytest.mark.parametrize("seed", range(10))
def test_steps_in_place(seed):
    rng = random.Random(100 + seed)
    state = random_state(rng, rng.randint(1, 30), 150, 8, 16)
    new = [rng.choice([0, 1, 1, 17]) for _ in state.pages]
    a, _ = step(state, None, new, in_place=True, source_given=False)
    b, _ = step(state, None, new, source_given=False)
    want, rows, pairs, _ = state.step(list(range(len(new))), new)
    same(a, want, rows, pairs, in_place=True)
    same(b, want, rows, pairs)


@pytest.mark.parametrize("B,n_pages", [(1, 1), (513, 3000), (1024, 20001)])
def test_many_requests_and_pages(B, n_pages):
    rng = random.Random(B)
    state = random_state(rng, B, n_pages, 5, 16)
    for r in rng.sample(range(n_pages), n_pages // 3):
        state.refs[r] += 1
    source = [rng.randrange(-1, B) if rng.random() < 0.5 else b for b in range(B)]
    new = [rng.choice([0, 1, 1, 1, 30]) for _ in source]
    a, _ = step(state, source, new)
    want, rows, pairs, _ = state.step(source, new)
    same(a, want, rows, pairs)


def test_all_requests_share_one_page_and_write_into_it():
    B = 700
    state = po.Pages([[3, 5]] * B, [20] * B, [0, 0, 0, B, 0, B] + [0] * 1000, 16, 4)
    a, st = step(state, list(range(B)), [1] * B)
    want, rows, pairs, _ = state.step(list(range(B)), [1] * B)
    same(a, want, rows, pairs)
    assert st == 0 and int(a["n_pairs"]) == B - 1  # the last one keeps it
    state.refs[5] += 1  # and somebody else holds it: all copy
    a, _ = step(state, list(range(B)), [1] * B)
    want, rows, pairs, _ = state.step(list(range(B)), [1] * B)
    same(a, want, rows, pairs)
    assert int(a["n_pairs"]) == B


def test_pages_that_run_out_serve_requests_in_order():
    state = po.Pages([[0], [1], [2], [3]], [16, 16, 10, 16], [1, 1, 1, 1, 0, 1, 0], 16, 4)
    a, st = step(state, [0, 1, 2, 3], [17, 1, 3, 1])
    want, rows, pairs, short = state.step([0, 1, 2, 3], [17, 1, 3, 1])
    same(a, want, rows, pairs)
    assert short and st == 3 and want.lengths == [33, 16, 13, 16]
    freed, st = step(state, [0, 1, 2, -1], [17, 1, 3, 0])  # what is freed is there at once
    assert st == 0 and freed["lengths_out"].tolist() == [33, 17, 13, 0] and freed["table_out"][1, 1] == 6


def test_bad_sources_lengths_and_offsets():
    state = po.Pages([[0], [1], [2], [3]], [16, 16, 10, 16], [1, 1, 1, 1, 0, 0, 0], 16, 4)
    a, st = step(state, [0, 4, 2, -2], [1, 1, 1, 1])
    assert st == fsx.FSX_ERR_DEVICE_ARG
    assert a["lengths_out"].tolist()[0] == 17 and a["lengths_out"].tolist()[2] == 11
    assert a["refs_out"].tolist()[:4] == [1, 1, 1, 0]  # page 1, freed by its request, is the lowest free one for request 0
    assert a["lengths_out"].tolist() == [17, 0, 11, 0] and a["rows"].tolist()[1::2] == [-1, -1]
    state.lengths[1] = 65  # more than its table holds
    a, st = step(state, [0, 1, 2, 3], [1, 1, 1, 1])
    assert st == fsx.FSX_ERR_DEVICE_ARG and a["lengths_out"].tolist() == [17, 0, 11, 17] and a["rows"].tolist()[1] == -1
    state.lengths[1], state.pages[2] = 16, [99]  # a last page that is none of the cache
    a, st = step(state, [0, 1, 2, 3], [1, 1, 1, 1])
    assert st == fsx.FSX_ERR_DEVICE_ARG and a["lengths_out"].tolist() == [17, 17, 10, 17]
    state.pages[2] = [2]
    table, lengths, refs, st = table_of(state), ints(state.lengths, torch.int64), ints(state.refs), status()
    rows, pairs, n = ints([55] * 3, torch.int64), ints([[0, 0]] * 4), ints([0])
    for bad in ([0, 1, 2, 3, 4], [0, 2, 1, 2, 3], [-1, 0, 1, 2, 3]):  # past the rows, back, negative
        st.zero_()
        fsx.pages_step(table.clone(), lengths.clone(), refs, ints(bad, torch.int64), 16, torch.empty_like(table), torch.empty_like(lengths),
                       torch.empty_like(refs), rows, pairs, n, st)
        assert int(st) == fsx.FSX_ERR_DEVICE_ARG


def test_no_new_rows():
    state = po.Pages([[0], [1]], [16, 3], [1, 2, 0], 16, 2)
    a, st = step(state, [1, 1, 0], [0, 0, 0])
    want, rows, pairs, _ = state.step([1, 1, 0], [0, 0, 0])
    same(a, want, rows, pairs)
    assert st == 0 and rows == []


def test_a_step_is_captured_and_replayed_in_place():
    state = po.Pages([[0], [1], []], [16, 3, 0], [1, 1] + [0] * 30, 16, 6)
    table, lengths, refs, new = table_of(state), ints(state.lengths, torch.int64), ints(state.refs), [1, 1, 1]
    rows, pairs, n, st = torch.empty(3, dtype=torch.int64, device="cuda"), ints([[0, 0]] * 3), ints([0]), status()
    at = offsets(new)
    args = (table, lengths, refs, at, 16, table, lengths, refs, rows, pairs, n, st)
    saved = [x.clone() for x in (table, lengths, refs)]
    fsx.pages_step(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fsx.pages_step(*args)
    for x, y in zip((table, lengths, refs), saved):
        x.copy_(y)
    for _ in range(20):
        graph.replay()
        state, want, _, _ = state.step([0, 1, 2], new)
        assert rows.tolist() == want
    assert lengths.tolist() == state.lengths == [36, 23, 20] and refs.tolist() == state.refs and int(st) == 0


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(12))
def test_compaction_of_random_states(seed, in_place):
    rng = random.Random(seed)
    n_pages = rng.choice([1, 2, 7, 100, 3001, 9000])
    state = random_state(rng, rng.randint(1, 300), n_pages, 9, 16)
    for b in range(len(state.pages)):  # some have gone
        if rng.random() < 0.4:
            for p in state.pages[b][:state.need(state.lengths[b])]:
                state.refs[p] -= 1
            state.lengths[b] = 0
    table, lengths, refs, st = table_of(state), ints(state.lengths, torch.int64), ints(state.refs), status()
    pairs, n = torch.full((n_pages // 2 + 1, 2), 55, dtype=torch.int32, device="cuda"), ints([55])
    table_out, refs_out = (table, refs) if in_place else (torch.full_like(table, 55), torch.full_like(refs, 55))
    before = table.cpu().tolist()
    fsx.pages_compact(table, lengths, refs, 16, table_out, refs_out, pairs, n, st)
    want, moves = state.compact()
    assert int(st) == 0 and int(n) == len(moves) and [tuple(p) for p in pairs[:len(moves)].tolist()] == moves
    assert (pairs[len(moves):] == 55).all() and refs_out.tolist() == want.refs
    for b, (got, row) in enumerate(zip(table_out.cpu().tolist(), want.pages)):
        k = state.need(state.lengths[b])
        assert got[:k] == row[:k] and got[k:] == before[b][k:]


def test_compaction_reports_bad_entries():
    table, refs = ints([[0, 7, 99, 5], [-1, 3, 3, 3]]), ints([1, 0, 0, 1, 0, 1, 0, 1])
    pairs, n, st, out, refs_out = ints([[0, 0]] * 4), ints([0]), status(), torch.empty_like(table), torch.empty_like(refs)
    fsx.pages_compact(table, ints([64, 32], torch.int64), refs, 16, out, refs_out, pairs, n, st)
    assert int(st) == fsx.FSX_ERR_DEVICE_ARG and out.tolist() == [[0, 2, 99, 1], [-1, 3, 3, 3]]
    assert refs_out.tolist() == [1, 1, 1, 1, 0, 0, 0, 0] and pairs[:int(n)].tolist() == [[5, 1], [7, 2]]


@pytest.mark.parametrize("page_rows,kv_heads,layers", [(16, 1, 1), (16, 8, 3), (64, 3, 2), (1024, 2, 1), (16, 300, 1), (512, 20, 1)])
def test_copies_of_every_plane(page_rows, kv_heads, layers):
    n_pages, g = 21, torch.Generator(device="cuda").manual_seed(1)
    rows = n_pages * page_rows
    caches = [torch.randn(rows, kv_heads, 128, device="cuda", generator=g).bfloat16() for _ in range(layers)] + \
             [torch.randint(0, 127, (rows, kv_heads, 128), device="cuda", generator=g, dtype=torch.uint8) for _ in range(layers)]
    scales = [torch.randn(kv_heads, rows, device="cuda", generator=g) for _ in range(layers)]
    bounds = [torch.randint(-9, 9, (n_pages, kv_heads, 2, 128), device="cuda", generator=g).to(torch.int8)]
    bound_scales = [torch.randn(kv_heads, n_pages, device="cuda", generator=g)]
    planes = fsx.page_planes(page_rows, caches, scales, bounds, bound_scales)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(2)).int()
    pairs, n, st = order[:20].view(10, 2).cuda(), ints([7]), status()

    def pages(t):  # [pages, ...]
        return t.view(n_pages, page_rows, kv_heads, 128) if t.dim() == 3 else t if t.dim() == 4 else \
            t.view(kv_heads, n_pages, -1).transpose(0, 1)

    everything = caches + scales + bounds + bound_scales
    want = [t.clone() for t in everything]
    for t in want:
        pages(t)[pairs[:7, 1].long()] = pages(t)[pairs[:7, 0].long()].clone()
    fsx.pages_copy(planes, pairs, n, st)
    assert int(st) == 0 and all(torch.equal(a, b) for a, b in zip(everything, want))
    fsx.pages_copy(planes, pairs[:0], n, st)
    n.zero_()
    fsx.pages_copy(planes, pairs.flip(1).contiguous(), n, st)
    assert int(st) == 0 and all(torch.equal(a, b) for a, b in zip(everything, want))
    bad = torch.tensor([[0, 21], [-1, 3], [5, 6]], dtype=torch.int32, device="cuda")
    n.fill_(3)
    fsx.pages_copy(planes, bad, n, st)
    for t in want:
        pages(t)[6] = pages(t)[5]
    assert int(st) == fsx.FSX_ERR_DEVICE_ARG and all(torch.equal(a, b) for a, b in zip(everything, want))
    for count in (-1, 4):
        st.zero_()
        n.fill_(count)
        fsx.pages_copy(planes, bad, n, st)
        assert int(st) == fsx.FSX_ERR_DEVICE_ARG and all(torch.equal(a, b) for a, b in zip(everything, want))


def test_copies_of_unaligned_planes_and_of_many():
    flat = torch.arange(1000, dtype=torch.int32, device="cuda")
    st, planes = status(), fsx.PagePlanes([fsx.PagePlane(flat.data_ptr() + 4, 12, 0, 1)], 30, [flat])
    want = flat.clone()
    want[1 + 3 * 7:1 + 3 * 8] = flat[1 + 3 * 2:1 + 3 * 3]
    fsx.pages_copy(planes, ints([[2, 7]]), ints([1]), st)
    assert torch.equal(flat, want) and int(st) == 0
    tensors = [torch.full((32, 1, 128), float(i), dtype=torch.bfloat16, device="cuda") for i in range(512)]
    for i, t in enumerate(tensors):
        t[16:] = -i
    fsx.pages_copy(fsx.page_planes(16, tensors), ints([[1, 0]]), ints([1]), st)
    assert all((t == -i).all() for i, t in enumerate(tensors)) and int(st) == 0
