"""fsx_page_bounds and fsx_page_select on the GPU: every code, scale and choice equal to the oracle's."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle, pages_oracle as po
from paper_2607_15621_gb300 import fsx

from llm_cases import normal, to64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def tables(lens, page_rows, seed, spare=2, more=2):
    need = [-(-n // page_rows) for n in lens]
    order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).int()
    table, at = torch.full((len(lens), max(need) + more), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def key_cache(rows, kv_heads, kind, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, kv_heads, 128, generator=g) * torch.exp(torch.randn(rows, kv_heads, 1, generator=g))
    if kind == "e4m3":
        code, s = llm_oracle.cache_write(to64(x.to(BF)))
        return torch.from_numpy(code).float().to(torch.float8_e4m3fn).cuda(), torch.from_numpy(s).float().T.contiguous().cuda(), code * s[..., None]
    x = x.to(kind)
    return x.cuda(), None, to64(x)


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", [BF, HF, "e4m3"])
@pytest.mark.parametrize("page_rows,kv_heads", [(16, 1), (16, 3), (32, 8), (128, 2)])
def test_bounds(page_rows, kv_heads, kind):
    lens = [1, page_rows, 0, 3 * page_rows + 1, 4 * page_rows - 1]
    table, n_pages = tables(lens, page_rows, page_rows)
    cache, scale, value = key_cache(n_pages * page_rows, kv_heads, kind, kv_heads)
    cache = cache.clone()
    if kind != "e4m3":
        cache[int(table[0, 0]) * page_rows + 1:(int(table[0, 0]) + 1) * page_rows] = math.nan  # behind the request's only row
    for start in (None, [0, 0, 0, 3 * page_rows, 2 * page_rows + 5]):
        bounds = torch.full((n_pages, kv_heads, 2, 128), 55, dtype=torch.int8, device="cuda")
        bound_scale, st = torch.full((kv_heads, n_pages), 7.0, device="cuda"), status()
        fsx.page_bounds(cache, table.cuda(), torch.tensor(lens, device="cuda"), page_rows, bounds, bound_scale, st, k_scale=scale,
                        start=None if start is None else torch.tensor(start, device="cuda"))
        assert int(st) == 0
        want, want_scale = np.full((n_pages, kv_heads, 2, 128), 55), np.full((kv_heads, n_pages), 7.0)
        for b, n in enumerate(lens):
            for j in range((start or [0] * 5)[b] // page_rows, -(-n // page_rows)):
                p = int(table[b, j])
                for h in range(kv_heads):
                    rows = slice(p * page_rows, p * page_rows + min(page_rows, n - j * page_rows))
                    want[p, h], want_scale[h, p] = po.page_bounds(value[rows, h])
        assert np.array_equal(bounds.cpu().numpy(), want) and np.array_equal(bound_scale.double().cpu().numpy(), want_scale)


def test_bounds_at_the_borders_of_the_scale():
    x = torch.zeros(9 * 16, 1, 128)
    for p, top in enumerate([127, 127.5, 63.5, 63.75, 2.0 ** -126, 2.0 ** -133, 3e38, 1.0, 0]):
        x[p * 16 + 3, 0, 5], x[p * 16 + 9, 0, 77] = top, -top / 3
        x[p * 16 + 4, 0, 6] = 1e-30 * min(top, 1)
    x = x.to(BF)
    bounds, bs, st = torch.empty(9, 1, 2, 128, dtype=torch.int8, device="cuda"), torch.empty(1, 9, device="cuda"), status()
    fsx.page_bounds(x.cuda(), torch.arange(9, dtype=torch.int32, device="cuda")[None], torch.tensor([144], device="cuda"), 16, bounds, bs, st)
    assert int(st) == 0
    for p in range(9):
        want, s = po.page_bounds(to64(x)[p * 16:p * 16 + 16, 0])
        assert np.array_equal(bounds[p, 0].cpu().numpy(), want) and float(bs[0, p]) == s


@pytest.mark.parametrize("kind", [BF, HF, "e4m3"])
def test_bounds_leave_out_what_is_not_finite(kind):
    cache, scale, value = key_cache(48, 2, kind, 1)
    value = value.copy()
    wild = [(3, 0, 7, math.nan), (20, 1, 64, math.nan), (33, 0, 0, math.nan)]
    if kind != "e4m3":
        wild += [(5, 0, 7, math.inf), (21, 1, 9, -math.inf)]
        cache[:16, 1, 100] = math.inf  # a dimension without a finite key
        value[:16, 1, 100] = math.inf
    if kind == "e4m3":
        bits = cache.view(torch.uint8)
        for r, h, d, _ in wild:
            bits[r, h, d] = 0xff
    else:
        for r, h, d, y in wild:
            cache[r, h, d] = y
    for r, h, d, y in wild:
        value[r, h, d] = y
    bounds, bs, st = torch.empty(3, 2, 2, 128, dtype=torch.int8, device="cuda"), torch.empty(2, 3, device="cuda"), status()
    fsx.page_bounds(cache, torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([48], device="cuda"), 16, bounds, bs, st,
                    k_scale=scale)
    assert int(st) == fsx.FSX_ERR_RANGE
    for p in range(3):
        for h in range(2):
            want, s = po.page_bounds(value[p * 16:p * 16 + 16, h])
            assert np.array_equal(bounds[p, h].cpu().numpy(), want) and float(bs[h, p]) == s


def test_bounds_of_bad_pages_and_lengths_are_left_out():
    cache, _, value = key_cache(64, 1, BF, 2)
    table = torch.tensor([[0, 4], [1, -1], [2, 3], [3, 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([32, 32, 33, 16], device="cuda")  # pages 4 and -1 are none; more rows than the table holds
    bounds, bs, st = torch.full((4, 1, 2, 128), 55, dtype=torch.int8, device="cuda"), torch.full((1, 4), 7.0, device="cuda"), status()
    fsx.page_bounds(cache, table, lens, 16, bounds, bs, st)
    assert int(st) == fsx.FSX_ERR_DEVICE_ARG
    for p in (0, 1, 3):
        assert np.array_equal(bounds[p, 0].cpu().numpy(), po.page_bounds(value[p * 16:p * 16 + 16, 0])[0])
    assert (bounds[2] == 55).all() and float(bs[0, 2]) == 7
    st = status()
    fsx.page_bounds(cache, table[3:], lens[3:], 16, bounds, bs, st, start=torch.tensor([-1], device="cuda"))
    assert int(st) == fsx.FSX_ERR_DEVICE_ARG


class Choice:
    def __init__(self, lens, heads, kv_heads, page_rows, seed, dtype=BF, spread=1.0, more=2):
        g = torch.Generator().manual_seed(seed)
        self.table, n = tables(lens, page_rows, seed, more=more)
        self.lens, self.page_rows, self.kv_heads = lens, page_rows, kv_heads
        self.bounds = torch.randint(-127, 128, (n, kv_heads, 2, 128), generator=g).sort(2)[0].to(torch.int8)
        self.scale = 2.0 ** torch.randint(-2, 2, (kv_heads, n), generator=g)
        self.q = normal(g, len(lens), heads, 128, dtype=dtype, scale=spread)
        self.status = status()

    def run(self, most, first=1, last=1, q=None):
        picked = torch.full((len(self.lens), self.kv_heads, most), 77, dtype=torch.int32, device="cuda")
        fsx.page_select(self.q.cuda() if q is None else q, self.bounds.cuda(), self.scale.cuda(), self.table.cuda(),
                        torch.tensor(self.lens, device="cuda"), self.page_rows, picked, self.status, first=first, last=last)
        return picked.cpu().tolist()

    def want(self, most, first=1, last=1):
        g = self.q.shape[1] // self.kv_heads
        out = []
        for b, n in enumerate(self.lens):
            pages = self.table[b, :-(-n // self.page_rows)].long()
            out.append([])
            for h in range(self.kv_heads):
                took = list(range(len(pages)))
                if len(pages) > most:
                    took = po.page_select(po.page_scores(to64(self.q[b, h * g:(h + 1) * g]), self.bounds[pages, h].numpy().astype(np.int64),
                                                         self.scale[h, pages].double().numpy()), first, last, most)
                out[-1].append(took + [-1] * (most - len(took)))
        return out


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (4, 4), (10, 2), (64, 1)])
def test_selection(heads, kv_heads, dtype):
    c = Choice([0, 1, 16, 17, 400, 1601], heads, kv_heads, 16, heads, dtype)
    for most, first, last in ((1, 0, 0), (1, 1, 0), (2, 1, 1), (7, 1, 1), (26, 2, 3), (101, 0, 1), (300, 1, 1)):
        assert c.run(most, first, last) == c.want(most, first, last)
    assert int(c.status) == 0


@pytest.mark.parametrize("pages,requests", [(1000, 1), (3000, 1), (700, 40)])
def test_selection_over_clusters(pages, requests):
    lens = [pages * 16 - 3 * b for b in range(requests)]
    c = Choice(lens, 4, 2, 16, pages)
    for most in (3, 64, 511):
        assert c.run(most) == c.want(most)


def test_selection_of_few_pages_in_a_wide_table():
    c = Choice([5 * 16, 900, 0, 70 * 16], 4, 2, 16, 3, more=5000)
    assert c.run(8) == c.want(8)


def test_ties_go_to_the_lowest_page():
    c = Choice([64 * 40, 64 * 300], 4, 2, 64, 1)
    c.bounds[:] = c.bounds[0]
    c.scale[:] = 1
    assert c.run(9) == c.want(9) == [[list(range(8)) + [39]] * 2, [list(range(8)) + [299]] * 2]
    c.q[:] = 0
    assert c.run(9, 0, 0) == [[list(range(9))] * 2] * 2


def test_scores_of_every_size_and_sign():
    c = Choice([16 * 200], 2, 1, 16, 5)
    c.bounds[:] = -c.bounds.abs()
    c.bounds = c.bounds.sort(2)[0]
    c.scale[:] = 2.0 ** torch.randint(-126, 120, c.scale.shape, generator=torch.Generator().manual_seed(6)).float()
    assert c.run(50) == c.want(50)
    c.q = c.q.abs()
    assert c.run(50) == c.want(50)


def test_queries_that_are_not_finite_and_bad_pages():
    c = Choice([16 * 30, 16 * 30], 4, 2, 16, 8)
    c.q[0, 1, 5], c.q[0, 3, 9] = math.inf, math.nan
    assert c.run(6) == c.want(6) and int(c.status) == fsx.FSX_ERR_RANGE
    c = Choice([16 * 30, -1, 16 * 90], 4, 2, 16, 8, more=0)
    c.lens[2] = 16 * 91
    c.table[0, 12] = 1 << 20
    got = c.run(6)
    assert int(c.status) == fsx.FSX_ERR_DEVICE_ARG and got[1:] == [[[-1] * 6] * 2] * 2
    c.status.zero_()
    assert all(12 not in x for x in got[0]) and all(x == sorted(set(x)) and len(x) == 6 for x in got[0])


def test_selection_is_captured_and_replayed():
    c = Choice([16 * 100] * 3, 4, 2, 16, 9)
    q, picked = c.q.cuda(), torch.zeros(3, 2, 12, dtype=torch.int32, device="cuda")
    args = (c.bounds.cuda(), c.scale.cuda(), c.table.cuda(), torch.tensor(c.lens, device="cuda"), 16, picked, c.status)
    fsx.page_select(q, *args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fsx.page_select(q, *args)
    c.q = -c.q
    q.neg_()
    graph.replay()
    assert picked.cpu().tolist() == c.want(12)


def test_bounds_of_codes_whose_scales_are_far_apart_or_no_powers_of_two():
    """Rows of a page with scales that one fp16 unit holds, and with scales that it does not."""
    g = torch.Generator().manual_seed(4)
    code = torch.from_numpy(llm_oracle.E4M3[:127])[torch.randint(0, 127, (6 * 64, 1, 128), generator=g)] * (torch.randint(0, 2, (6 * 64, 1, 128), generator=g) * 2 - 1)
    scale = torch.ones(6 * 64, 1)
    scale[64:128] = 2.0 ** torch.randint(-7, 8, (64, 1), generator=g)    # 14 powers: just held
    scale[128:192] = 2.0 ** torch.randint(-8, 8, (64, 1), generator=g)   # 15
    scale[192:256] = 2.0 ** torch.randint(-120, 100, (64, 1), generator=g)
    scale[256:320] = torch.rand(64, 1, generator=g) + 0.01
    scale[320 + 40] = 2.0 ** 13  # late in the page: the ends so far change their unit
    cache = code.float().to(torch.float8_e4m3fn).cuda()
    bounds, bs, st = torch.empty(6, 1, 2, 128, dtype=torch.int8, device="cuda"), torch.empty(1, 6, device="cuda"), status()
    for start in (None, torch.zeros(1, dtype=torch.int64, device="cuda")):  # a warp a page, eight warps a page
        fsx.page_bounds(cache, torch.arange(6, dtype=torch.int32, device="cuda")[None], torch.tensor([6 * 64 - 5], device="cuda"), 64, bounds, bs,
                        st, k_scale=scale.T.contiguous().cuda(), start=start)
        assert int(st) == 0
        value = to64(cache) * scale.double().numpy()[..., None]
        value = value.astype(np.float32).astype(np.float64)  # codes times scales are fp32
        for p in range(6):
            want, s = po.page_bounds(value[p * 64:min(p * 64 + 64, 6 * 64 - 5), 0])
            assert np.array_equal(bounds[p, 0].cpu().numpy(), want) and float(bs[0, p]) == s


@pytest.mark.parametrize("pages", [300, 2500])
def test_many_pages_at_the_border(pages):
    """Scores that one page far above squeezes into few digits: hundreds at the border, told apart by their last bits or not at all."""
    c = Choice([16 * pages] * 2, 2, 1, 16, 10)
    g = torch.Generator().manual_seed(11)
    c.q[:] = 1
    c.bounds[:] = 0
    c.bounds[:, 0, 1, 0] = 127
    c.bounds[:, 0, 1, 1:9] = torch.randint(0, 3, (len(c.bounds), 8), generator=g).to(torch.int8)
    c.scale[:] = 2.0 ** -30
    c.scale[0, c.table[0, 5]] = 2.0 ** 30
    c.bounds[c.table[1, 40]] = -1  # and one below zero
    for most in (3, 100, pages // 2, pages - 1):
        assert c.run(most) == c.want(most)
        assert c.run(most, 0, 0) == c.want(most, 0, 0)
