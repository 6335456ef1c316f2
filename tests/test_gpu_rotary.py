"""fsx_rotary on the GPU against the fp64 oracle, and its cache rows against fsx_cache_write_e4m3.

Bound of a value: its own rounding (half a step of the type, 2^-25 at least for fp16's subnormals) and fp32 products of
cosines and sines: the angle is off by 2^-32 of a turn, its fp32 half turn by 2^-25, sincospi by 2 units, the products and their sum by
one rounding each: 2^-20 (|a| + |b|) holds all of them.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from paper_2607_15621_gb300 import fsx

from llm_cases import U, normal, to64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def near(got, x, want, dtype, adjacent):
    y = np.abs(x)
    both = y[..., 0::2] + y[..., 1::2] if adjacent else y[..., :64] + y[..., 64:]
    both = np.repeat(both, 2, -1) if adjacent else np.concatenate([both, both], -1)
    err = np.abs(to64(got) - want)
    assert (err <= U[dtype] * np.abs(want) + 2.0 ** -20 * both + 2.0 ** -25).all()


def inputs(n, heads, kv_heads, dtype, seed, axes=1, far=5000):
    g = torch.Generator().manual_seed(seed)
    buf = normal(g, n, heads + 2 * kv_heads, 128, dtype=dtype).cuda()
    pos = torch.randint(-far, far, (axes, n), generator=g)
    return buf[:, :heads], buf[:, heads:heads + kv_heads], buf[:, heads + kv_heads:], pos.cuda()


def caches(rows, kv_heads, kind):
    if kind == "e4m3":
        return ([torch.full((rows, kv_heads, 128), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv"],
                [torch.full((kv_heads, rows), 7.0, device="cuda") for _ in "kv"])
    return [torch.full((rows, kv_heads, 128), 7.0, dtype=kind, device="cuda") for _ in "kv"], [None, None]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,heads,kv_heads,sections", [(1, 1, 1, (64,)), (1, 32, 32, (64,)), (3, 5, 1, (16, 24, 24)), (33, 8, 2, (32, 32)),
                                                       (130, 12, 4, (1, 0, 60, 3)), (7, 28, 4, (64,))])
def test_queries_and_keys(n, heads, kv_heads, sections, dtype, adjacent):
    q, k, _, pos = inputs(n, heads, kv_heads, dtype, n, len(sections))
    pairs = fsx.rotary_pairs(sections, adjacent=adjacent)
    qo, ko, st = torch.full_like(q, 7).contiguous(), torch.full_like(k, 7).contiguous(), status()
    fsx.rotary(q, k, pos, pairs, st, q_out=qo, k_out=ko)
    assert int(st) == 0
    for x, y in ((q, qo), (k, ko)):
        near(y, to64(x), po.rotary(to64(x), pos.cpu().numpy(), list(pairs.axis), list(pairs.rate), adjacent), dtype, adjacent)
    only_q, only_k = torch.empty_like(qo), torch.empty_like(ko)
    fsx.rotary(q, None, pos, pairs, st, q_out=only_q)
    fsx.rotary(None, k, pos, pairs, st, k_out=only_k)
    assert torch.equal(only_q, qo) and torch.equal(only_k, ko)
    fsx.rotary(q, k, pos, pairs, st, q_out=q, k_out=k)  # in place, columns of one buffer
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("kind", ["e4m3", "same"])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,kv_heads", [(1, 32), (5, 3), (64, 8), (301, 2)])
def test_cache_rows_are_those_of_a_cache_write(n, kv_heads, dtype, kind):
    q, k, v, pos = inputs(n, 2 * kv_heads, kv_heads, dtype, n + 7, 2)
    pairs = fsx.rotary_pairs((40, 24), per_axis=True)
    kind = dtype if kind == "same" else kind
    m = n + 40
    rows = torch.randperm(m, generator=torch.Generator().manual_seed(n))[:n].cuda()
    qo, ko, st = torch.empty_like(q).contiguous(), torch.empty_like(k).contiguous(), status()
    (kc, vc), (ks, vs) = caches(m, kv_heads, kind)
    fsx.rotary(q, k, pos, pairs, st, q_out=qo, k_out=ko, v=v, rows=rows, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs)
    near(ko, to64(k), po.rotary(to64(k), pos.cpu().numpy(), list(pairs.axis), list(pairs.rate)), dtype, False)
    (kd, vd), (kt, vt) = caches(m, kv_heads, kind)
    if kind == "e4m3":
        fsx.cache_write(ko, v.contiguous(), rows, kd, vd, kt, vt, st)
        assert torch.equal(ks, kt) and torch.equal(vs, vt)
        kc, vc, kd, vd = (x.view(torch.uint8) for x in (kc, vc, kd, vd))
    else:
        kd[rows], vd[rows] = ko, v
    assert torch.equal(kc, kd) and torch.equal(vc, vd) and int(st) == 0
    # without k_out, and without queries, the same cache
    (ke, ve), (ku, vu) = caches(m, kv_heads, kind)
    fsx.rotary(None, k, pos, pairs, st, v=v, rows=rows, k_cache=ke, v_cache=ve, k_scale=ku, v_scale=vu)
    same = (lambda a, b: torch.equal(a.view(torch.uint8), b)) if kind == "e4m3" else torch.equal
    assert same(ke, kc) and same(ve, vc)


def test_far_positions_keep_their_angle():
    pos = [0, 1, 123456, 10 ** 6 + 1, 2 ** 24 + 1, 2 ** 31 - 1, -(2 ** 31)]
    g = torch.Generator().manual_seed(3)
    q = normal(g, len(pos), 2, 128, dtype=HF).cuda()
    at = torch.tensor([pos], device="cuda")
    rate = [1.0, -1.0, 0.0, 1e-9, 37.5, 1000.0, 3.14159, 0.5] * 8
    pairs, out = fsx.RotaryPairs([0] * 64, rate), torch.empty_like(q)
    fsx.rotary(q, None, at, pairs, status(), q_out=out)
    # angles by whole numbers: pos * rate exactly, reduced by 2 pi to 80 digits
    from decimal import Decimal, getcontext
    getcontext().prec = 80
    pi2 = Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563281257241799726")
    x, want = to64(q), np.empty(q.shape)
    for r, p in enumerate(pos):
        for j in range(64):
            t = float(Decimal(p) * Decimal(rate[j]) % pi2)
            want[r, :, j] = x[r, :, j] * math.cos(t) - x[r, :, j + 64] * math.sin(t)
            want[r, :, j + 64] = x[r, :, j] * math.sin(t) + x[r, :, j + 64] * math.cos(t)
    near(out, x, want, HF, False)


def test_values_that_are_not_finite_and_rows_outside_the_cache():
    q, k, v, pos = inputs(4, 4, 2, BF, 11)
    pos.zero_()
    k[1, 0, 5], v[2, 1, 127], k[3, 1, 64] = math.inf, math.nan, -math.inf
    (kc, vc), (ks, vs) = caches(20, 2, "e4m3")
    (kd, vd), (kt, vt) = caches(20, 2, "e4m3")
    ko, st, other = torch.empty_like(k).contiguous(), status(), status()
    rows = torch.tensor([3, 0, 19, 7], device="cuda")
    fsx.rotary(None, k, pos, fsx.rotary_pairs(), st, k_out=ko, v=v, rows=rows, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs)
    assert int(st) == fsx.FSX_ERR_RANGE
    fsx.cache_write(ko, v.contiguous(), rows, kd, vd, kt, vt, other)
    assert int(other) == fsx.FSX_ERR_RANGE
    for a, b in ((kc, kd), (vc, vd)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(ks, kt) and torch.equal(vs, vt)
    for kind in ("e4m3", BF):
        for bad in (-1, 20, 1 << 40):
            (kc, vc), (ks, vs) = caches(20, 2, kind)
            clean, st = [c.clone() for c in (kc, vc)], status()
            rows = torch.tensor([3, bad, 19, 7], device="cuda")
            fsx.rotary(None, v, pos, fsx.rotary_pairs(), st, k_out=ko, v=v, rows=rows, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs)
            assert int(st) == fsx.FSX_ERR_DEVICE_ARG
            changed = [(a.view(torch.uint8) != b.view(torch.uint8)).flatten(1).any(1).nonzero().flatten().tolist() for a, b in zip((kc, vc), clean)]
            assert changed == [[3, 7, 19], [3, 7, 19]]
            assert torch.equal(ko[1], v[1])  # the keys themselves are written all the same


def test_strides_none_rows_another_stream_and_a_graph():
    q, k, v, pos = inputs(70, 8, 2, BF, 21)
    pairs, st = fsx.rotary_pairs(), status()
    qo, ko = torch.empty_like(q).contiguous(), torch.empty_like(k).contiguous()
    fsx.rotary(q, k, pos, pairs, st, q_out=qo, k_out=ko)
    wide = torch.full((70, 13, 128), 7.0, dtype=BF, device="cuda")
    fsx.rotary(q.contiguous(), k.contiguous(), pos, pairs, st, q_out=wide[:, 1:9], k_out=wide[:, 10:12])
    assert torch.equal(wide[:, 1:9], qo) and torch.equal(wide[:, 10:12], ko)
    assert (wide[:, [0, 9, 12]] == 7).all()
    fsx.rotary(q[:0], k[:0], pos[:, :0].contiguous(), pairs, st, q_out=qo[:0], k_out=ko[:0])
    side, again = torch.cuda.Stream(), torch.zeros_like(qo)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fsx.rotary(q, None, pos, pairs, st, q_out=again)
    side.synchronize()
    assert torch.equal(again, qo)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fsx.rotary(q, k, pos, pairs, st, q_out=again, k_out=ko)
    pos.neg_()
    graph.replay()
    fsx.rotary(q, None, pos, pairs, st, q_out=qo)
    assert torch.equal(again, qo) and int(st) == 0


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("kind", [None, "e4m3", BF])
@pytest.mark.parametrize("n,heads,kv_heads", [(30001, 2, 1), (30001, 5, 1), (13000, 1, 1), (1301, 32, 8), (3001, 16, 4), (1001, 40, 8)])
def test_many_rows_are_what_few_of_them_are(n, heads, kv_heads, kind, adjacent):
    """Several rows a warp, whole rows a warp and rows shared out over warps give the same bits."""
    q, k, v, pos = inputs(n, heads, kv_heads, BF, heads, 3, far=100000)
    pairs = fsx.rotary_pairs((16, 24, 24), adjacent=adjacent)
    m = n + 11
    rows = torch.randperm(m, generator=torch.Generator().manual_seed(n))[:n].cuda()
    rows[n // 2] = -1  # one that has no place

    def run(parts):
        qo, ko, st = torch.empty_like(q).contiguous(), torch.empty_like(k).contiguous(), status()
        (kc, vc), (ks, vs) = caches(m, kv_heads, kind) if kind else ([None, None], [None, None])
        for a in range(0, n, parts):
            b = min(n, a + parts)
            write = dict(v=v[a:b], rows=rows[a:b], k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs) if kind else {}
            fsx.rotary(q[a:b], k[a:b], pos[:, a:b].contiguous(), pairs, st, q_out=qo[a:b], k_out=ko[a:b], **write)
        assert int(st) == (fsx.FSX_ERR_DEVICE_ARG if kind else 0)
        return [qo, ko] + [x.view(torch.uint8) for x in (kc, vc, ks, vs) if x is not None]

    whole, few = run(n), run(97)
    assert all(torch.equal(a, b) for a, b in zip(whole, few))
    some = torch.arange(0, n, n // 7, device="cuda")
    near(whole[0][some], to64(q[some]), po.rotary(to64(q[some]), pos[:, some].cpu().numpy(), list(pairs.axis), list(pairs.rate), adjacent), BF, adjacent)
