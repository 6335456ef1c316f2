"""The documented sequence over a cache in pages, word for word: requests that fork, grow over a page's end, are freed."""
from __future__ import annotations

import os
import re

import pytest
import torch

from oracle import pages_oracle as po
from paper_2607_15621_gb300 import fsx

from llm_cases import check, normal, to64

pytestmark = pytest.mark.gpu

DOCUMENT = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def ints(v, t=torch.int32):
    return torch.tensor(v, dtype=t, device="cuda")


def test_the_sequence_over_pages():
    code = next(x for x in re.findall(r"```python\n(.*?)```", open(DOCUMENT).read(), re.S) if "pages_step" in x)
    g = torch.Generator().manual_seed(6)
    P, n_pages, heads, hk, width = 16, 40, 8, 2, 8
    lengths, new, source = [30, 17, 64, 5], [1, 20, 0, 1], [0, 0, -1, 2]
    held = [-(-n // P) for n in lengths]
    order, at = torch.randperm(n_pages, generator=g).tolist(), 0
    table = [[-1] * width for _ in lengths]
    for b, n in enumerate(held):
        table[b][:n] = order[at:at + n]
        at += n
    refs = [0] * n_pages
    for p in order[:at]:
        refs[p] = 1
    k_cache, v_cache = (normal(g, n_pages * P, hk, 128).cuda() for _ in "kv")
    qkv = normal(g, sum(new), heads + 2 * hk, 128).cuda()
    B = len(new)
    bounds, bound_scale = torch.zeros(n_pages, hk, 2, 128, dtype=torch.int8, device="cuda"), torch.ones(hk, n_pages, device="cuda")
    status = ints([0])
    fsx.page_bounds(k_cache, ints(table), ints(lengths, torch.int64), P, bounds, bound_scale, status)
    names = dict(torch=torch, page_rows=P, k_cache=k_cache, v_cache=v_cache, table=ints(table), lengths=ints(lengths, torch.int64),
                 refs=ints(refs), new_offsets=ints([0] + new, torch.int64).cumsum(0), table2=ints([[0] * width] * B),
                 lengths2=ints([0] * B, torch.int64), rows=ints([0] * sum(new), torch.int64), copies=ints([[0, 0]] * B), n_copies=ints([0]),
                 status=status, source=ints(source), q=qkv[:, :heads], k=qkv[:, heads:heads + hk], v=qkv[:, heads + hk:], B=B, heads=heads,
                 kv_heads=hk, positions=torch.randint(0, 99, (3, sum(new)), generator=g).cuda(), bounds=bounds, bound_scale=bound_scale,
                 picked=torch.zeros(B, hk, 3, dtype=torch.int32, device="cuda"), out=torch.zeros(B, heads, 128, dtype=torch.bfloat16, device="cuda"))
    exec(compile("from paper_2607_15621_gb300 import fsx\n" + code, DOCUMENT, "exec"), names)
    assert int(status) == 0
    table2, lengths2 = names["table2"], names["lengths2"]
    assert lengths2.tolist() == [31, 50, 0, 65]
    again, scale = torch.zeros_like(bounds), torch.ones_like(bound_scale)
    fsx.page_bounds(k_cache, table2, lengths2, P, again, scale, status)
    mine = torch.cat([row[:-(-n // P)] for row, n in zip(table2.cpu(), lengths2.tolist())]).long().cuda()
    assert torch.equal(bounds[mine], again[mine]) and torch.equal(bound_scale[:, mine], scale[:, mine])  # none of them is stale
    newest = names["q"][names["new_offsets"][1:] - 1]
    want, _ = po.paged_attention(to64(newest), to64(k_cache), to64(v_cache), table2.tolist(), lengths2.tolist(), P, names["picked"].cpu().numpy())
    check(names["out"], None, want, None, torch.bfloat16, float(v_cache.abs().max()))
