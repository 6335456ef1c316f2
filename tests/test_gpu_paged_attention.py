"""fsx_paged_attention on the GPU against the fp64 oracle (bounds: llm_cases)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle, pages_oracle as po
from paper_2607_15621_gb300 import fsx

from llm_cases import check, normal, to64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def coded(x):
    """Codes as values and powers of two as scales that hold the rows, whatever they are: for caches of many rows."""
    s = 2.0 ** (torch.frexp(x.float().abs().amax(-1))[1].double() - 8)
    return (x.double() / s[..., None]).float().to(torch.float8_e4m3fn).double().numpy(), s.numpy()


class Case:
    """Requests over a cache of shuffled pages; every row that belongs to none is NaN."""

    def __init__(self, lens, heads, kv_heads, page_rows, dtype, cache, seed, spare=3, width=None, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        B, self.page_rows = len(lens), page_rows
        need = [-(-n // page_rows) for n in lens]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).int()
        width = width or max(1, max(need) + 2)
        table, at = torch.full((B, width), -1, dtype=torch.int32), 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        rows = self.n_pages * page_rows
        used = torch.zeros(rows, dtype=torch.bool)
        for b, n in enumerate(lens):
            used[torch.from_numpy(po.rows_of(table[b].tolist(), n, page_rows))] = True
        self.lens, self.table, self.lengths = list(lens), table.cuda(), torch.tensor(lens, device="cuda")
        self.q = normal(g, B, heads, 128, dtype=dtype, scale=scale).cuda()
        kv = [normal(g, rows, kv_heads, 128, dtype=dtype) for _ in "kv"]
        if cache == "e4m3":
            self.cache, self.scale, self.value = [], [], []
            for x in kv:
                code, s = llm_oracle.cache_write(to64(x)) if rows * kv_heads < 50000 else coded(x)
                code[~used.numpy()] = math.nan
                s[~used.numpy()] = math.nan
                self.value.append(code * s[..., None])
                self.cache.append(torch.from_numpy(code).float().to(torch.float8_e4m3fn).cuda())
                self.scale.append(torch.from_numpy(s).float().T.contiguous().cuda())
        else:
            for x in kv:
                x[~used] = math.nan
            self.cache, self.scale, self.value = [x.cuda() for x in kv], [None, None], [to64(x) for x in kv]
        self.out = torch.full((B, heads, 128), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((heads, B), 7.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.workspace = torch.zeros(fsx.paged_attention_workspace_bytes(B, heads, kv_heads), dtype=torch.uint8, device="cuda")

    def run(self, **over):
        a = dict(q=self.q, k_cache=self.cache[0], v_cache=self.cache[1], table=self.table, lengths=self.lengths, page_rows=self.page_rows,
                 out=self.out, status=self.status, workspace=self.workspace, k_scale=self.scale[0], v_scale=self.scale[1], lse=self.lse)
        return fsx.paged_attention(**dict(a, **over))

    def want(self, picked=None):
        return po.paged_attention(to64(self.q), *self.value, self.table.tolist(), self.lens, self.page_rows, picked)

    def compare(self, picked=None, scale=1.0):
        want, lse = self.want(picked)
        check(self.out, self.lse, want, lse, self.q.dtype, np.nanmax(np.abs(self.value[1]), initial=1.0), scale)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (6, 2), (8, 1), (9, 1), (16, 1), (34, 2), (64, 1)])
def test_heads(heads, kv_heads, dtype, cache):
    c = Case([1, 0, 15, 16, 17, 130], heads, kv_heads, 16, dtype, dtype if cache == "same" else cache, heads)
    c.run()
    assert int(c.status) == 0
    c.compare()
    assert (c.out[1] == 0).all() and torch.isneginf(c.lse[:, 1]).all()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("page_rows", [16, 32, 64, 128, 1024])
def test_lengths_where_steps_chunks_and_pages_end(page_rows, cache):
    lens = [1, 15, 16, 31, 33, 63, 64, 65, 127, 129, 511, 512, 513, 575, 1023, 1025]
    c = Case(lens, 4, 2, page_rows, BF, BF if cache == "same" else cache, page_rows)
    c.run()
    assert int(c.status) == 0
    c.compare()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("lens,heads,kv_heads", [([5000], 2, 2), ([20000], 8, 1), ([3000, 0, 700, 9001], 20, 2), ([2100] * 3, 3, 3)])
def test_long_histories_that_are_cut(lens, heads, kv_heads, cache):
    c = Case(lens, heads, kv_heads, 32, HF, HF if cache == "same" else cache, len(lens))
    c.run()
    assert int(c.status) == 0
    c.compare()
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(3):  # the same bits, whichever CTA joins
        c.out.fill_(7)
        c.run()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)


def test_more_requests_than_a_warp_and_the_most_of_them():
    g = torch.Generator().manual_seed(5)
    for B in (33, 300, 1024):
        lens = torch.randint(0, 40, (B,), generator=g).tolist()
        c = Case(lens, 2, 1, 16, BF, "e4m3", B)
        c.run()
        assert int(c.status) == 0
        c.compare()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("page_rows,most", [(16, 1), (16, 7), (64, 5), (256, 3)])
def test_picked_pages(page_rows, most, cache):
    lens = [1, page_rows, 3 * page_rows + 5, 9 * page_rows, 20 * page_rows - 1, 0]
    c = Case(lens, 8, 2, page_rows, BF, BF if cache == "same" else cache, most)
    g = torch.Generator().manual_seed(most)
    picked = torch.full((len(lens), 2, most), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        pages = -(-n // page_rows)
        for h in range(2):
            take = torch.randperm(pages, generator=g)[:most]  # in any order, the last page among them or not
            picked[b, h, :len(take)] = take.int()
    picked[4, 1, most // 2] = -1  # one that names none
    c.run(picked=picked.cuda())
    assert int(c.status) == 0
    c.compare(picked.numpy())


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("B,heads,kv_heads", [(310, 1, 1), (160, 20, 2), (100, 8, 4)])
def test_many_items_some_of_them_cut(B, heads, kv_heads, cache):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 1100, (B,), generator=g).tolist()
    lens[7] = 2900
    c = Case(lens, heads, kv_heads, 64, BF, BF if cache == "same" else cache, B)
    c.run()
    assert int(c.status) == 0
    c.compare()
    first = c.out.clone()
    for _ in range(3):
        c.out.fill_(7)
        c.run()
        assert torch.equal(c.out, first)
    page = int(c.table[7, 30])
    c.table[7, 30] = -1  # in one of several pieces: the others' results are as before
    c.out.fill_(7)
    c.run()
    assert int(c.status) == fsx.FSX_ERR_DEVICE_ARG and (c.out[7] == 7).all()
    c.out[7], c.table[7, 30] = first[7], page
    assert torch.equal(c.out, first)


def test_picked_none_gives_zeros():
    c = Case([100, 50], 4, 2, 16, BF, BF, 1)
    c.run(picked=torch.full((2, 2, 4), -1, dtype=torch.int32, device="cuda"))
    assert int(c.status) == 0 and (c.out == 0).all() and torch.isneginf(c.lse).all()


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("bad", [-1, -5, 1 << 30, "n_pages"])
def test_bad_pages_are_reported_and_their_request_is_left_out(bad, cache):
    lens = [40, 3000, 200, 17]
    c = Case(lens, 4, 2, 16, BF, BF if cache == "same" else cache, 3)
    c.table[1, 150] = c.n_pages if bad == "n_pages" else bad  # in one of several pieces
    c.table[2, 12] = c.n_pages if bad == "n_pages" else bad   # the last page
    c.table[3, 2] = c.n_pages if bad == "n_pages" else bad    # behind the last page: not read
    c.run()
    assert int(c.status) == fsx.FSX_ERR_DEVICE_ARG
    assert (c.out[1:3] == 7).all() and (c.lse[:, 1:3] == 7).all()
    c.table[1, 150] = c.table[2, 12] = 0
    want, lse = c.want()
    want[1:3], lse[:, 1:3] = math.nan, math.nan
    check(c.out, c.lse, want, lse, BF, np.nanmax(np.abs(c.value[1])))


def test_bad_lengths_and_bad_picks():
    c = Case([40, 30, 100, 17], 4, 2, 16, HF, HF, 4)
    c.lengths[1], c.lengths[2] = -1, c.table.shape[1] * 16 + 1
    c.run()
    assert int(c.status) == fsx.FSX_ERR_DEVICE_ARG and (c.out[1:3] == 7).all() and not (c.out[[0, 3]] == 7).any()
    c = Case([40, 30, 100, 17], 4, 2, 16, HF, HF, 4)
    picked = torch.tensor([[[0, 1]] * 2, [[1, 0]] * 2, [[0, 7], [3, 6]], [[-2, 0], [1, -1]]], dtype=torch.int32, device="cuda")
    c.run(picked=picked)  # request 2 has 7 pages, 3 has 2
    assert int(c.status) == fsx.FSX_ERR_DEVICE_ARG
    assert (c.out[2, :2] == 7).all() and (c.out[3, :2] == 7).all() and not (c.out[2, 2:] == 7).any() and not (c.out[3, 2:] == 7).any()
    assert not (c.out[:2] == 7).any()


@pytest.mark.parametrize("scale", [1e-4, 1.0, 30.0])
def test_flat_and_steep_softmax(scale):
    c = Case([900, 64], 8, 2, 64, BF, "e4m3", 9, scale=scale)
    c.run()
    c.compare(scale=scale)


def test_infinities_that_are_seen_are_carried():
    c = Case([50, 50], 2, 1, 16, BF, BF, 8)
    row = int(po.rows_of(c.table[0].tolist(), 50, 16)[20])
    c.cache[1][row, 0, 3] = math.inf
    c.run()
    assert torch.isinf(c.out[0, :, 3]).all() and c.out[0, :, [2, 4]].isfinite().all() and c.out[1].isfinite().all()


def test_shared_pages_strided_queries_another_stream_and_graphs_in_turn():
    c = Case([500, 300, 77], 8, 2, 32, BF, BF, 12)
    c.table[1, :9] = c.table[0, :9]  # a fork
    buf = torch.zeros(3, 12, 128, dtype=BF, device="cuda")
    buf[:, 3:11] = c.q
    c.run(q=buf[:, 3:11])
    c.lens[1], want = 288, None
    c.lengths[1] = 288
    c.run(q=buf[:, 3:11])
    c.compare()
    want = c.out.clone()
    c.out.fill_(7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    side.synchronize()
    assert torch.equal(c.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    c.lengths.copy_(torch.tensor([33, 64, 5]))  # what a graph replays follows the tensors
    c.lens = [33, 64, 5]
    for _ in range(3):
        graph.replay()
    c.compare()
    assert int(c.status) == 0


def test_rows_beyond_32_bits_of_bytes():
    rows = (1 << 31) // (32 * 128) + 64 * 20  # 4.3 GB in 16 bits
    rows -= rows % 64
    cache = torch.zeros(rows, 32, 128, dtype=HF, device="cuda")
    g = torch.Generator().manual_seed(2)
    last = normal(g, 128, 32, 128, dtype=HF)
    cache[-128:] = last.cuda()
    q = normal(g, 1, 32, 128, dtype=HF).cuda()
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(fsx.paged_attention_workspace_bytes(1, 32, 32), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[rows // 64 - 1, rows // 64 - 2]], dtype=torch.int32, device="cuda")
    fsx.paged_attention(q, cache, cache, table, torch.tensor([100], device="cuda"), 64, out, status, ws)
    value = np.concatenate([to64(last)[64:], to64(last)[:36]])
    want, _ = po.paged_attention(to64(q), value, value, [[0, 1]], [100], 64)
    check(out, None, want, None, HF, np.abs(value).max())
    assert int(status) == 0
