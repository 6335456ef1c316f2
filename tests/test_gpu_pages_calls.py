"""Calls of the operators over pages that tests of one operator do not make: tensors elsewhere, graphs of all of them, two streams."""
from __future__ import annotations

import pytest
import torch

from paper_2607_15621_gb300 import fsx

pytestmark = pytest.mark.gpu

B, HEADS, KV, P, PAGES, WIDTH = 5, 8, 2, 16, 60, 8


class Step:
    """One decoding step: tables, rotary positions, bounds, selection, attention, compaction, on buffers of its own."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        z = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device="cuda")
        self.k, self.v = (torch.randn(PAGES * P, KV, 128, generator=g).bfloat16().cuda() for _ in "kv")
        self.lengths0 = torch.tensor([100, 17, 0, 64, 33])
        order = torch.randperm(PAGES, generator=g)[:B * WIDTH].int().view(B, WIDTH)
        self.table0 = torch.where(torch.arange(WIDTH) * P < self.lengths0[:, None], order, -1).int()
        self.refs0 = torch.zeros(PAGES, dtype=torch.int32)
        self.refs0[self.table0[self.table0 >= 0].long()] = 1
        self.table, self.lengths, self.refs = z(B, WIDTH), z(B, dtype=torch.int64), z(PAGES)
        self.new = torch.arange(B + 1, device="cuda")
        self.rows, self.pairs, self.moves, self.n = z(B, dtype=torch.int64), z(B, 2), z(PAGES // 2, 2), z(1)
        self.qkv0 = torch.randn(B, HEADS + 2 * KV, 128, generator=g).bfloat16()
        self.qkv = self.qkv0.cuda()
        self.bounds, self.bs = z(PAGES, KV, 2, 128, dtype=torch.int8), torch.ones(KV, PAGES, device="cuda")
        self.picked, self.out, self.status = z(B, KV, 4), torch.zeros(B, HEADS, 128, dtype=torch.bfloat16, device="cuda"), z(1)
        self.ws = z(fsx.paged_attention_workspace_bytes(B, HEADS, KV), dtype=torch.uint8)
        self.planes = fsx.page_planes(P, [self.k, self.v], bounds=[self.bounds], bound_scales=[self.bs])
        self.turn = fsx.rotary_pairs()
        self.reset()

    def reset(self):
        for to, what in ((self.table, self.table0), (self.lengths, self.lengths0), (self.refs, self.refs0), (self.qkv, self.qkv0)):
            to.copy_(what)

    def run(self):
        q, k, v = self.qkv[:, :HEADS], self.qkv[:, HEADS:HEADS + KV], self.qkv[:, HEADS + KV:]
        fsx.pages_step(self.table, self.lengths, self.refs, self.new, P, self.table, self.lengths, self.refs, self.rows, self.pairs, self.n, self.status)
        fsx.pages_copy(self.planes, self.pairs, self.n, self.status)
        fsx.rotary(q, k, self.lengths[None], self.turn, self.status, q_out=q, v=v, rows=self.rows, k_cache=self.k, v_cache=self.v)
        fsx.page_bounds(self.k, self.table, self.lengths, P, self.bounds, self.bs, self.status)
        fsx.page_select(q, self.bounds, self.bs, self.table, self.lengths, P, self.picked, self.status)
        fsx.paged_attention(q, self.k, self.v, self.table, self.lengths, P, self.out, self.status, self.ws, picked=self.picked)
        fsx.pages_compact(self.table, self.lengths, self.refs, P, self.table, self.refs, self.moves, self.n, self.status)
        fsx.pages_copy(self.planes, self.moves, self.n, self.status)

    def state(self):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        return [x.clone() for x in (self.out, self.picked, self.table, self.refs, self.lengths, self.k, self.bounds)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_whole_step_is_captured_and_two_run_at_once():
    steps = [Step(1), Step(2)]
    want = []
    for s in steps:
        s.run()
        s.reset()
        s.run()
        s.run()
        want.append(s.state())
    again = [Step(1), Step(2)]
    for s in again:
        s.run()
        s.reset()
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in again]
    for _ in range(2):
        for s, stream in zip(again, side):
            with torch.cuda.stream(stream):
                s.run()
    torch.cuda.synchronize()
    assert all(equal(s.state(), w) for s, w in zip(again, want))
    third = Step(1)
    third.run()
    third.reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third.run()
    third.reset()
    graph.replay()
    graph.replay()
    assert equal(third.state(), want[0])


def test_tensors_elsewhere_are_refused():
    s = Step(3)
    host = torch.zeros(1, dtype=torch.int32)
    q, k = s.qkv[:, :HEADS], s.qkv[:, HEADS:HEADS + KV]
    calls = [lambda: fsx.rotary(q.cpu(), k, s.lengths[None], s.turn, s.status, q_out=q, k_out=k),
             lambda: fsx.rotary(q, k, s.lengths[None], s.turn, host, q_out=q, k_out=k),
             lambda: fsx.paged_attention(q, s.k, s.v.cpu(), s.table, s.lengths, P, s.out, s.status, s.ws),
             lambda: fsx.paged_attention(q, s.k, s.v, s.table, s.lengths, P, s.out, s.status, s.ws.cpu()),
             lambda: fsx.page_bounds(s.k, s.table0, s.lengths, P, s.bounds, s.bs, s.status),
             lambda: fsx.page_select(q, s.bounds, s.bs, s.table, s.lengths.cpu(), P, s.picked, s.status),
             lambda: fsx.pages_step(s.table, s.lengths, s.refs0, s.new, P, s.table, s.lengths, s.refs, s.rows, s.pairs, s.n, s.status),
             lambda: fsx.pages_compact(s.table, s.lengths, s.refs, P, s.table, s.refs, s.moves.cpu(), s.n, s.status),
             lambda: fsx.pages_copy(s.planes, s.pairs, s.n.cpu(), s.status),
             lambda: fsx.pages_copy(fsx.page_planes(P, [s.k.cpu()]), s.pairs, s.n, s.status)]
    for call in calls:
        with pytest.raises(fsx.FsxError, match="current device"):
            call()
    with pytest.raises(fsx.FsxError):
        fsx.page_planes(P, [s.k, s.v.cpu()])
    assert int(s.status) == 0
