"""fsx_paged_attention's weights: an output is rounded once, by its own type, and nothing of the weights' rounding shows.

Values are +1 and -1, as many of each in every dimension, and weights nearly equal, so that an output is the small difference of
sums of magnitude A = 1: its own rounding, U |y| (half a step: 2^-8 of bf16, 2^-11 of fp16), no longer hides the rounding of the weights.

Bound, times A: weights in two parts of the product's type leave the second part's rounding, 2^-8 2^-8 of bf16 and 2^-11 2^-11 of
fp16; a score is an fp32 sum of 128 products, 128 2^-23 sum|q k| / sqrt(128) < 2^-18 at |q| about 2^-8; exponential 2^-21; the
sums over at most 320 keys are fewer than 64 fp32 additions, 64 2^-23 = 2^-17. Together below 2^-16 for products in fp16 (over 8-bit
caches, and of fp16) and 2^-15 in bf16. One part alone leaves 2^-12 / sqrt(3 n) of fp16 on average over n keys, 2^-9 / sqrt(3 n) of
bf16, and several times that at the worst of thousands of outputs.
"""
from __future__ import annotations

import pytest
import torch

from oracle import llm_oracle, pages_oracle as po
from paper_2607_15621_gb300 import fsx

from llm_cases import U, normal, to64

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("picked", [False, True])
@pytest.mark.parametrize("repeat", [1, 40])  # a line of few items, a queue of many
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (24, 2)])
@pytest.mark.parametrize("dtype,cache", [(BF, "same"), (HF, "same"), (BF, "e4m3"), (HF, "e4m3")])
def test_the_weights_rounding_does_not_show(dtype, cache, heads, kv_heads, repeat, picked):
    lens = [16, 34, 64, 100, 320] * repeat
    g = torch.Generator().manual_seed(heads + repeat)
    need = [-(-n // 16) for n in lens]
    rows, width = 16 * sum(need), max(need)
    table, at = torch.zeros(len(lens), width, dtype=torch.int32), 0
    k, v = normal(g, rows, kv_heads, 128, dtype=dtype), torch.zeros(rows, kv_heads, 128, dtype=dtype)
    for b, n in enumerate(lens):
        table[b, :need[b]] = torch.arange(at, at + need[b])
        half = torch.rand(n, kv_heads, 128, generator=g).argsort(0) < n // 2
        v[16 * at:16 * at + n] = torch.where(half, 1.0, -1.0).to(dtype)
        at += need[b]
    q = normal(g, len(lens), heads, 128, dtype=dtype, scale=2.0 ** -8)
    if cache == "e4m3":
        codes = [llm_oracle.cache_write(to64(x)) for x in (k, v)]
        values = [c * s[..., None] for c, s in codes]
        caches = [torch.from_numpy(c).float().to(torch.float8_e4m3fn).cuda() for c, _ in codes]
        scales = [torch.from_numpy(s).float().T.contiguous().cuda() for _, s in codes]
    else:
        values, caches, scales = [to64(x) for x in (k, v)], [k.cuda(), v.cuda()], [None, None]
    out, st = torch.empty(len(lens), heads, 128, dtype=dtype, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(fsx.paged_attention_workspace_bytes(len(lens), heads, kv_heads), dtype=torch.uint8, device="cuda")
    pick = torch.arange(width - 1, -1, -1, dtype=torch.int32).expand(len(lens), kv_heads, width).clone() if picked else None
    if picked:  # all pages of each request, the last one first
        for b, n in enumerate(need):
            pick[b, :, :n], pick[b, :, n:] = torch.arange(n - 1, -1, -1, dtype=torch.int32), -1
        pick = pick.cuda()
    fsx.paged_attention(q.cuda(), *caches, table.cuda(), torch.tensor(lens, device="cuda"), 16, out, st, ws, k_scale=scales[0],
                        v_scale=scales[1], picked=pick)
    want, _ = po.paged_attention(to64(q), *values, table.tolist(), lens, 16)
    slack = abs(to64(out) - want) - U[dtype] * abs(want) - 2.0 ** -25
    print("slack %.3g" % slack.max())
    assert int(st) == 0 and slack.max() <= (2.0 ** -15 if dtype == BF and cache == "same" else 2.0 ** -16)


@pytest.mark.parametrize("repeat", [1, 60])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_infinite_scales_of_values_are_carried(dtype, repeat):
    """A value is its code times its row's scale: infinite, or NaN where the code is 0."""
    n, B = 50, 2 * repeat
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randint(1, 60, (64, 4, 128), generator=g, dtype=torch.uint8) for _ in "kv")  # positive codes
    v[:, 0, 3], v[7, 1, 5] = 0, 0x80 | 9
    ks, vs = torch.full((4, 64), 0.25), torch.full((4, 64), 0.5)
    vs[:, 7], vs[2, 40] = float("inf"), float("inf")
    table = torch.arange(4, dtype=torch.int32).repeat(B, 1)
    lengths = torch.tensor([n, 7] * repeat)  # every second request ends before that row
    out, st = torch.empty(B, 8, 128, dtype=dtype, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = normal(g, B, 8, 128, dtype=dtype)
    ws = torch.zeros(fsx.paged_attention_workspace_bytes(B, 8, 4), dtype=torch.uint8, device="cuda")
    f8 = lambda x: x.cuda().view(torch.float8_e4m3fn)
    fsx.paged_attention(q.cuda(), f8(k), f8(v), table.cuda(), lengths.cuda(), 16, out, st, ws, k_scale=ks.cuda(), v_scale=vs.cuda())
    got = out.float().cpu().view(B, 4, 2, 128)
    assert int(st) == 0 and got[1::2].isfinite().all()
    got = got[0::2]
    assert got[:, 0, :, 3].isnan().all() and (got[:, 1, :, 5] == -float("inf")).all()
    got[:, 0, :, 3], got[:, 1, :, 5] = float("inf"), float("inf")
    assert (got == float("inf")).all()
