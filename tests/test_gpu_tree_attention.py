"""fsx_tree_attention on the GPU against the fp64 oracle: 16-bit and 8-bit caches, trees, single tokens, ragged ends."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import llm_oracle
from paper_2607_15621_gb300 import fsx

from llm_cases import check, normal, offsets, to64

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def tree_masks(new, rng):
    words = []
    for n in new:
        mine = []
        for i in range(n):
            parent = int(rng.integers(-1, i)) if i else -1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        words += mine
    return words


def make(lens, new, heads=4, kv_heads=2, dtype=BF16, cache8=True, seed=0, scale=1.0, gap=3, poison=True):
    """Requests with `gap` free rows (NaN) in front of and behind every cache range."""
    gen, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    starts = np.cumsum([gap] + [n + gap for n in lens])[:-1].astype(np.int64)
    rows = int(sum(lens) + gap * (len(lens) + 1))
    total = sum(new)
    c = dict(q=normal(gen, total, heads, 128, dtype=dtype, scale=scale).cuda(),
             kn=normal(gen, total, kv_heads, 128, dtype=dtype).cuda(), vn=normal(gen, total, kv_heads, 128, dtype=dtype).cuda(),
             no=offsets(new), mask=tree_masks(new, rng), starts=starts, off=offsets(lens), lens=list(lens), ks=None, vs=None)
    own = np.zeros(rows, bool)
    for s, n in zip(starts, lens):
        own[s:s + n] = True
    free = torch.as_tensor(~own)
    k, v = (normal(gen, rows, kv_heads, 128, dtype=dtype) for _ in "kv")
    if cache8:
        c["kc"], c["vc"] = (torch.zeros(rows, kv_heads, 128, dtype=torch.float8_e4m3fn, device="cuda") for _ in "kv")
        c["ks"], c["vs"] = (torch.empty(kv_heads, rows, device="cuda") for _ in "kv")
        fsx.cache_write(k.cuda(), v.cuda(), None, c["kc"], c["vc"], c["ks"], c["vs"],
                        torch.zeros(1, dtype=torch.int32, device="cuda"))
        if poison:
            for t in (c["kc"], c["vc"]):
                t.view(torch.uint8)[free.cuda()] = 0x7f
            for t in (c["ks"], c["vs"]):
                t[:, free.cuda()] = math.nan
    else:
        if poison:
            k[free], v[free] = math.nan, math.inf
        c["kc"], c["vc"] = k.cuda(), v.cuda()
    return c


def space(c):
    n = fsx.tree_attention_workspace_bytes(len(c["lens"]), c["q"].shape[0], c["q"].shape[1], c["kn"].shape[1])
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def run(c, lse=True, workspace=None, stream=None, starts=True):
    out = torch.full(c["q"].shape, 7.0, dtype=c["q"].dtype, device="cuda")
    z = torch.full((c["q"].shape[1], c["q"].shape[0]), 7.0, device="cuda") if lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int64), device="cuda")
    words = [w - (1 << 64) if w >> 63 else w for w in c["mask"]]
    fsx.tree_attention(c["q"], c["kn"], c["vn"], dev(c["no"]), dev(words), c["kc"], c["vc"], dev(c["off"]), out, status,
                       space(c) if workspace is None else workspace, k_scale=c["ks"], v_scale=c["vs"],
                       starts=dev(c["starts"]) if starts else None, lse=z, stream=stream)
    torch.cuda.synchronize()
    return out, z, int(status)


def caches64(c):
    if c["ks"] is None:
        return to64(c["kc"]), to64(c["vc"])
    return tuple(to64(x) * to64(s).T[..., None] for x, s in ((c["kc"], c["ks"]), (c["vc"], c["vs"])))


def oracle(c):
    with np.errstate(invalid="ignore"):
        k, v = caches64(c)
        return llm_oracle.tree_attention(to64(c["q"]), to64(c["kn"]), to64(c["vn"]), c["no"], c["mask"], k, v, c["starts"],
                                         c["lens"])


def v_max(c):
    _, v = caches64(c)
    rows = np.concatenate([v[s:s + n] for s, n in zip(c["starts"], c["lens"])])
    vn = to64(c["vn"])
    return max(np.abs(rows).max(initial=0), np.abs(vn[np.isfinite(vn)]).max(initial=0))


def agree(c, scale=1.0, **kw):
    out, lse, status = run(c, **kw)
    assert status == fsx.FSX_OK
    want, want_lse = oracle(c)
    check(out, lse, want, want_lse, c["q"].dtype, v_max(c), scale)
    return out, lse


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("lens", [[0], [1, 0, 2], [63, 64, 65], [127, 128, 129], [300, 5, 700]])
def test_cache_lengths(lens, cache8, dtype):
    agree(make(lens, [3] * len(lens), dtype=dtype, cache8=cache8, seed=len(lens)))


@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("new", [[1, 1, 1], [0, 1, 2], [64, 63, 5], [17, 33, 48]])
def test_drafts(new, cache8):
    agree(make([70, 130, 9], new, cache8=cache8, seed=sum(new)))


@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("heads,kv_heads,n", [(1, 1, 64), (3, 3, 5), (7, 1, 19), (8, 1, 64), (6, 2, 43), (64, 1, 5)])
def test_grouped_heads(heads, kv_heads, n, cache8):
    agree(make([150, 40], [n, 1], heads=heads, kv_heads=kv_heads, cache8=cache8, seed=heads))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("cache8", [True, False])
def test_single_tokens_over_long_caches(cache8, dtype):
    """Ranges that many blocks share, beside short ones and empty ones."""
    agree(make([5000, 0, 1, 2047, 64], [1] * 5, heads=4, kv_heads=4, dtype=dtype, cache8=cache8, seed=20))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("heads,kv_heads,lens,new", [
    (8, 2, [6000, 4100, 5200, 7001], [8, 5, 7, 6]),        # 20 to 32 rows an item, dozens of chunks, cut items
    (8, 2, [3000] * 20 + [1500, 40, 0], [6] * 23),         # about as many items as SMs
    (4, 1, [9000, 130], [60, 64]),                         # items of 240 and 256 rows
    (32, 4, [700, 1300, 257] * 6, [4, 16, 40] * 6),        # short and long, few and many rows together
])
def test_many_rows_over_long_caches(heads, kv_heads, lens, new, cache8, dtype):
    """Pieces that start and end anywhere in an item; the oracle on a few heads and tokens of each request."""
    c = make(lens, new, heads=heads, kv_heads=kv_heads, dtype=dtype, cache8=cache8, seed=len(lens))
    out, lse, status = run(c)
    assert status == fsx.FSX_OK
    assert torch.equal(run(c)[0], out)
    g = heads // kv_heads
    k, v = caches64(c)
    for b in range(len(lens)):
        t0, t1 = int(c["no"][b]), int(c["no"][b + 1])
        for kvh in sorted({0, kv_heads - 1}):
            hs, tokens = [kvh * g, kvh * g + g - 1], sorted({t0, (t0 + t1) // 2, t1 - 1})
            for i in tokens:
                seen = [t0 + j for j in range(t1 - t0) if c["mask"][i] >> j & 1]
                rows = slice(c["starts"][b], c["starts"][b] + lens[b])
                kk = np.concatenate([k[rows, kvh], to64(c["kn"])[seen, kvh]])
                vv = np.concatenate([v[rows, kvh], to64(c["vn"])[seen, kvh]])
                for h in hs:
                    want, want_lse = llm_oracle.attention_row(to64(c["q"])[i, h], kk, vv)
                    check(out[i:i + 1, h:h + 1], lse[h:h + 1, i:i + 1], want[None, None], np.array([[want_lse]]), dtype,
                          np.abs(vv).max())


@pytest.mark.parametrize("cache8", [True, False])
def test_many_requests(cache8):
    rng = np.random.default_rng(21)
    lens, new = rng.integers(0, 90, 300), rng.integers(0, 4, 300)
    agree(make(lens.tolist(), new.tolist(), heads=2, kv_heads=1, cache8=cache8, seed=21))


@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("scale", [0.0, 8.0, 60.0])
def test_flat_and_sharp_scores(scale, cache8):
    agree(make([400, 64], [5, 9], cache8=cache8, seed=22, scale=scale), scale=scale)


@pytest.mark.parametrize("cache8", [True, False])
def test_rows_that_see_nothing_and_bits_past_the_tokens(cache8):
    c = make([0, 5, 0], [4, 4, 2], cache8=cache8, seed=23)
    c["mask"] = [0, 0b0010, 0, 0b1111, 0, 0, 0b1000, 0, 0, 1 << 63 | 0b100]
    agree(c)


def test_all_64_bits():
    c = make([40], [64], seed=24)
    c["mask"] = [(1 << 64) - 1 if i % 2 else 1 << 63 | 1 << i for i in range(64)]
    agree(c)


@pytest.mark.parametrize("cache8", [True, False])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_new_tokens_that_are_not_seen_have_no_effect(value, cache8):
    c = make([30, 200], [6, 40], cache8=cache8, seed=25)
    clean, lse, _ = run(c)
    for token in (2, 30):  # of requests 0 and 1
        c["kn"][token], c["vn"][token] = value, value
    out, lse2, status = run(c)
    assert status == fsx.FSX_OK
    blind = [i for i in range(46) if not (c["mask"][i] >> (2 if i < 6 else 24) & 1)]
    assert 2 not in blind and 30 not in blind and len(blind) > 10
    assert torch.equal(out[blind], clean[blind]) and torch.equal(lse[:, blind], lse2[:, blind])
    assert not torch.isfinite(out[2]).all() and not torch.isfinite(out[30]).all()


def test_a_large_spread_of_scales():
    """Scales of neighbouring rows 2^40 apart, as rows of very different size leave them."""
    c = make([200], [4], seed=26)
    f = torch.where(torch.arange(c["vs"].shape[1], device="cuda") % 3 == 0, 2.0 ** -40, 1.0)
    c["vs"] = c["vs"] * f
    c["ks"] = c["ks"] * f
    agree(c)


def test_scales_that_are_no_powers_of_two():
    c = make([200, 31], [4, 1], seed=27)
    c["ks"], c["vs"] = c["ks"] * 1.37, c["vs"] * 0.71
    agree(c)


@pytest.mark.parametrize("cache8", [True, False])
def test_without_starts_and_fused_columns(cache8):
    c = make([60, 130], [5, 20], heads=4, kv_heads=4, cache8=cache8, seed=28, gap=0)
    plain, lse, _ = run(c)
    rows = c["q"].shape[0]
    buf = torch.full((rows, 14 * 128 + 8), math.nan, dtype=BF16, device="cuda")
    for at, name in ((1, "q"), (5, "kn"), (10, "vn")):
        buf[:, at * 128:(at + 4) * 128] = c[name].reshape(rows, -1)
        c[name] = buf[:, at * 128:(at + 4) * 128].unflatten(1, (4, 128))
    out, lse2, status = run(c, starts=False)
    assert status == fsx.FSX_OK and torch.equal(out, plain) and torch.equal(lse, lse2)


@pytest.mark.parametrize("cache8", [True, False])
def test_a_workspace_serves_calls_of_other_shapes_and_streams(cache8):
    a = make([3000, 100], [2, 30], heads=8, kv_heads=2, cache8=cache8, seed=29)
    b = make([70] * 40, [1] * 40, heads=2, kv_heads=2, cache8=cache8, seed=30)
    ws = torch.zeros(max(space(a).numel(), space(b).numel()), dtype=torch.uint8, device="cuda")
    first = run(a, workspace=ws)[0]
    agree(b, workspace=ws)
    assert torch.equal(run(a, workspace=ws, stream=torch.cuda.Stream())[0], first)
    assert torch.equal(run(a, workspace=ws, lse=False)[0], first)


def test_a_bad_request_is_reported_and_passed_over():
    c = make([40, 30, 50], [3, 2, 4], seed=31)
    want, want_lse = oracle(c)
    rows = c["kc"].shape[0]
    bads = [dict(starts=np.array([c["starts"][0], -1, c["starts"][2]])),
            dict(starts=np.array([c["starts"][0], rows - 29, c["starts"][2]])),
            dict(starts=np.array([c["starts"][0], 1 << 40, c["starts"][2]]))]
    for bad in bads:
        out, lse, status = run(dict(c, **bad))
        assert status == fsx.FSX_ERR_DEVICE_ARG
        assert (out[3:5] == 7).all() and (lse[:, 3:5] == 7).all()
        for lo, hi in ((0, 3), (5, 9)):
            check(out[lo:hi], lse[:, lo:hi], want[lo:hi], want_lse[:, lo:hi], BF16, v_max(c))


def test_more_than_64_new_tokens_are_refused_on_the_device():
    c = make([10, 10], [64, 3], seed=32)
    c["no"] = np.array([0, 65, 67])
    out, _, status = run(c)
    assert status == fsx.FSX_ERR_DEVICE_ARG and (out[:65] == 7).all()


def test_offsets_beyond_32_bits():
    c = make([500], [3], heads=32, kv_heads=32, seed=33, gap=0)
    plain, lse, _ = run(c)
    rows = (1 << 32) // (32 * 128) + 700  # e4m3 caches of 4.3 GB
    for name in ("kc", "vc"):
        t = torch.empty(rows, 32, 128, dtype=torch.uint8, device="cuda")
        t[-500:] = c[name].view(torch.uint8)
        c[name] = t.view(torch.float8_e4m3fn)
    for name in ("ks", "vs"):
        t = torch.empty(32, rows, device="cuda")
        t[:, -500:] = c[name]
        c[name] = t
    c["starts"] = np.array([rows - 500])
    out, lse2, status = run(c)
    assert status == fsx.FSX_OK and torch.equal(out, plain) and torch.equal(lse, lse2)
