"""Operators over a cache in pages, as cases whose time and results can be measured.

Kinds of call (field "kind"):
  rotary  queries and keys turned by rotary positions of one or several axes (time, height, width), the keys and values
          written into the cache in the same pass (rotary)
  paged   one new token of each request over its pages, 16-bit or 8-bit (paged_attention)
  bounds  the bounds of all pages of prompts that have just been written (page_bounds)
  sparse  the same token over the few pages that a score selects: bounds of the newest page, selection, attention over the
          selected pages (page_bounds, page_select, paged_attention)
  step    a step of the page tables: requests forked, freed and grown, shared pages that would be written into copied
          over all layers (pages_step, pages_copy)
  compact pages in use moved to the front of the cache over all layers (pages_compact, pages_copy)

Shapes are the repository's own: 32 heads of 128 of a 7B-shaped backbone, also with grouped key/value heads, histories from
224 rows (64 instruction tokens and 40 frames x 4) to those of its sweep and far beyond, one vehicle to a fleet of 128.
Values follow the synthetic workloads: keys ~ N(0, 1) times a log-normal scale per head and dimension, queries and values
~ N(0, 1), rounded to the type.

A page is `page_rows` consecutive rows of a cache [rows, kv heads, 128]; 8-bit caches have e4m3 codes and one scale per
row and head, [kv heads, rows]. Request b's row j lies in page table[b, j // page_rows].
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
D = 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"bf16": 2, "fp16": 2, "e4m3": 1}


def listed():
    return [
        # one vehicle's next token on its way into the cache: latency
        dict(name="rotary_b1", kind="rotary", rows=1, far=4096, heads=32, kv_heads=32, dtype="bf16", cache="bf16", axes=1,
             adjacent=False, keys=False),
        # a fleet's next tokens into 8-bit pages, grouped heads, three axes
        dict(name="rotary_b128", kind="rotary", rows=128, far=131072, heads=32, kv_heads=8, dtype="bf16", cache="e4m3",
             axes=3, adjacent=False, keys=False),
        # the rows of a fleet's prompts; the prompt's attention reads the keys too
        dict(name="rotary_prompts_28001", kind="rotary", rows=28001, far=2048, heads=32, kv_heads=8, dtype="fp16",
             cache="fp16", axes=3, adjacent=True, keys=True),
        # one request over the cache as the append writes it, in small pages
        dict(name="paged_b1_224", kind="paged", batch=1, lo=224, hi=224, page_rows=16, heads=32, kv_heads=32, dtype="bf16",
             cache="bf16", lse=False),
        # a small fleet with long ragged histories, grouped heads
        dict(name="paged_b16_8192", kind="paged", batch=16, lo=1000, hi=8192, page_rows=64, heads=32, kv_heads=8,
             dtype="fp16", cache="fp16", lse=True),
        # the fleet batch of the benchmark, one token a vehicle, over 8-bit pages: the largest case
        dict(name="paged_b128_fleet", kind="paged", batch=128, lo=64, hi=2048, page_rows=32, heads=32, kv_heads=32,
             dtype="bf16", cache="e4m3", lse=False),
        # one request with a very long history, split over the whole GPU
        dict(name="paged_b1_131072", kind="paged", batch=1, lo=131072, hi=131072, page_rows=64, heads=32, kv_heads=8,
             dtype="bf16", cache="e4m3", lse=False),
        # bounds of a few long prompts' pages, once they are written
        dict(name="bounds_b4_32768", kind="bounds", batch=4, lo=20000, hi=32768, page_rows=32, kv_heads=8, cache="bf16"),
        # a small fleet that attends to at most 64 of its pages
        dict(name="sparse_b16_32768", kind="sparse", batch=16, lo=4096, hi=32768, page_rows=32, heads=32, kv_heads=8,
             dtype="bf16", cache="bf16", picked=64),
        # one request with a very long history over 8-bit pages
        dict(name="sparse_b1_131072", kind="sparse", batch=1, lo=131001, hi=131001, page_rows=64, heads=32, kv_heads=8,
             dtype="fp16", cache="e4m3", picked=96),
        # sixteen requests of four continuations each: the better ones forked, the others freed, all of them a token longer
        dict(name="step_b64", kind="step", batch=64, lo=200, hi=2000, page_rows=16, kv_heads=8, new=1, pages=8192, layers=4),
        # a cache of which half the requests have gone
        dict(name="compact_b48", kind="compact", batch=48, lo=200, hi=1000, page_rows=16, kv_heads=8, pages=4096, layers=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "paged", "paged", "paged", "bounds", "sparse", "sparse", "step", "compact"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if kv_heads * g <= 32])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    cache = rng.choice(["e4m3", dtype])
    page_rows = rng.choice([16, 16, 32, 64, 128])
    if kind == "rotary":
        rows = _log(rng, 1, 28000)
        cache = rng.choice([None, dtype, dtype] if rows > 512 else [None, dtype, "e4m3"])
        return dict(kind=kind, rows=rows, far=_log(rng, 64, 1000000), heads=heads, kv_heads=kv_heads, dtype=dtype, cache=cache,
                    axes=rng.choice([1, 2, 3]), adjacent=rng.random() < 0.3, keys=cache is None or rng.random() < 0.5)
    if kind in ("step", "compact"):
        batch = _log(rng, 2, 64)
        hi = _log(rng, 8, min(4000, 60000 // batch))
        case = dict(kind=kind, batch=batch, lo=max(1, _log(rng, max(1, hi // 16), hi)), hi=hi, page_rows=rng.choice([16, 32]),
                    kv_heads=rng.choice([1, 2, 8]), layers=rng.choice([1, 2, 4]))
        if kind == "step":
            case["new"] = _log(rng, 1, 40)
        # as many pages as the longest requests would need, and some
        case["pages"] = batch * (hi // case["page_rows"] + 4) + rng.randrange(8, 200)
        return case
    batch = _log(rng, 1, 128)
    hi = _log(rng, 1, min(131072, 131072 // batch * 2, 4000000 // (batch * kv_heads)))
    lo = max(0, _log(rng, max(1, hi // 16), hi) - 1)
    case = dict(kind=kind, batch=batch, lo=lo, hi=hi, page_rows=page_rows, heads=heads, kv_heads=kv_heads, dtype=dtype,
                cache=cache)
    if kind == "paged":
        case["lse"] = rng.random() < 0.3
    elif kind == "bounds":
        del case["heads"], case["dtype"]
    else:
        case["picked"] = _log(rng, 4, 128)
    return case


def _lengths(case):
    """Lengths of the case's requests: part of the case, not of the seed."""
    rng = random.Random("%d %d %d" % (case["batch"], case["lo"], case["hi"]))
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def _pages(n, page_rows):
    return -(-n // page_rows)


def _source(case):
    """step: whose pages each request takes on. Groups of four: two of them stay, one is forked from, one is freed."""
    rng = random.Random("%d %d %d source" % (case["batch"], case["lo"], case["hi"]))
    return [b if b % 4 < 2 else -1 if rng.random() < 0.1 else b - b % 4 + rng.randrange(2) for b in range(case["batch"])]


def _new(case):
    """step: new tokens of each request; freed ones get none."""
    rng = random.Random("%d %d %d new" % (case["batch"], case["lo"], case["hi"]))
    return [0 if s < 0 else rng.randint((case["new"] + 1) // 2, case["new"]) for s in _source(case)]


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _keys(gen, rows, heads):
    scale = torch.exp(0.5 * torch.randn(heads, D, generator=gen, device=DEV))
    return torch.randn(rows, heads, D, generator=gen, device=DEV) * scale


def _ints(v, t=torch.int64):
    return torch.tensor(v, dtype=t, device=DEV)


def _power(e):
    """2^e in 32 bits, exactly, for -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _least_power(top, most):
    """The smallest power of two s >= 2^-126 with top / s <= most (448 or 127, 2^8 or 2^6 times 1.75 or more); 1 for 0."""
    e = (torch.frexp(top)[1] - (9 if most == 448 else 7)).clamp(-126, 119)
    e = torch.where(top / _power(e) > most, e + 1, e)
    return torch.where(top > 0, _power(e), torch.ones_like(top))


def _codes(x):
    """e4m3 codes and scales of rows [..., 128] in 32 bits."""
    scale = _least_power(x.abs().amax(-1), 448)
    return (x / scale[..., None]).to(torch.float8_e4m3fn), scale


def _pairs(case):
    """Axis and rate (radians a position) of the 64 pairs of a head: sections of the pairs go to the axes."""
    n = case["axes"]
    sizes = {1: [64], 2: [32, 32], 3: [16, 24, 24]}[n]
    axis = [a for a, s in enumerate(sizes) for _ in range(s)]
    return sizes, axis, [10000.0 ** (-j / 64) for j in range(64)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    kind, hk = case["kind"], case["kv_heads"]
    if kind == "rotary":
        return _prepare_rotary(s, case, gen, seed)
    lens, p = _lengths(case), case["page_rows"]
    width = max(1, max(_pages(n, p) for n in lens) + 4)
    used = [_pages(n, p) for n in lens]
    if kind in ("step", "compact"):
        return _prepare_step(s, case, gen, lens, width)
    n_pages = sum(used) + 8
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    first = _ints(_offsets(used))
    j = torch.arange(width, device=DEV)
    table = torch.where(j < (first[1:] - first[:-1])[:, None], order[(first[:-1, None] + j).clamp(max=n_pages - 1)], -1)
    s.update(table=table.to(torch.int32), lengths=_ints(lens), most=max(max(lens), 1))
    rows = n_pages * p
    k = _keys(gen, rows, hk)
    if case["cache"] == "e4m3":
        k, sk = _codes(k)
        s["k_scale"] = sk.T.contiguous()
    else:
        k, s["k_scale"] = k.to(TYPES[case["cache"]]), None
    s["k_cache"] = k
    if kind in ("bounds", "sparse"):
        s["bounds"] = torch.zeros(n_pages, hk, 2, D, dtype=torch.int8, device=DEV)
        s["bound_scale"] = torch.ones(hk, n_pages, device=DEV)
    if kind == "bounds":
        return s
    v = torch.randn(rows, hk, D, generator=gen, device=DEV)
    if case["cache"] == "e4m3":
        v, sv = _codes(v)
        s["v_scale"] = sv.T.contiguous()
    else:
        v, s["v_scale"] = v.to(TYPES[case["cache"]]), None
    s["v_cache"] = v
    b, h, t = case["batch"], case["heads"], TYPES[case["dtype"]]
    s["q"] = torch.randn(b, h, D, generator=gen, device=DEV).to(t)
    s["out"] = torch.empty(b, h, D, dtype=t, device=DEV)
    s["lse"] = torch.empty(h, b, device=DEV) if case.get("lse") else None
    if kind == "sparse":
        s["picked"] = torch.empty(b, hk, case["picked"], dtype=torch.int32, device=DEV)
        s["newest"] = (s["lengths"] - 1).clamp(min=0)
        codes, scale = _bounds_of(s, torch.zeros_like(s["lengths"]))
        s["bounds"].copy_(codes)
        s["bound_scale"].copy_(scale)
    if own:
        from paper_2607_15621_gb300 import fsx
        s["workspace"] = torch.zeros(fsx.paged_attention_workspace_bytes(b, h, hk), dtype=torch.uint8, device=DEV)
    return s


def _prepare_rotary(s, case, gen, seed):
    n, h, hk, t = case["rows"], case["heads"], case["kv_heads"], TYPES[case["dtype"]]
    # q, k, v as the columns of one projection's output
    buf = torch.cat([torch.randn(n, h, D, generator=gen, device=DEV), _keys(gen, n, hk),
                     torch.randn(n, hk, D, generator=gen, device=DEV)], 1).to(t)
    sizes, axis, rate = _pairs(case)
    s.update(q=buf[:, :h], k=buf[:, h:h + hk], v=buf[:, h + hk:], axis=_ints(axis),
             rate=torch.tensor(rate, dtype=torch.float64, device=DEV),
             positions=torch.randint(0, case["far"], (case["axes"], n), generator=gen, device=DEV),
             q_out=torch.empty(n, h, D, dtype=t, device=DEV),
             k_out=torch.empty(n, hk, D, dtype=t, device=DEV) if case["keys"] else None)
    s["cache"], s["scale"] = [None, None], [None, None]
    if case["cache"]:
        m = (n + 300) // 16 * 16  # whole pages of 16 rows
        s["rows"] = torch.randperm(m, generator=gen, device=DEV)[:n]
        if case["cache"] == "e4m3":
            s["cache"] = [torch.zeros(m, hk, D, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in "kv"]
            s["scale"] = [torch.ones(hk, m, device=DEV) for _ in "kv"]
        else:
            s["cache"] = [torch.zeros(m, hk, D, dtype=t, device=DEV) for _ in "kv"]
    if own:
        from paper_2607_15621_gb300 import fsx
        s["pairs"] = fsx.rotary_pairs(sizes, adjacent=case["adjacent"])
    return s


def _prepare_step(s, case, gen, lens, width):
    p, n_pages, batch, kind = case["page_rows"], case["pages"], case["batch"], case["kind"]
    width += _pages(case.get("new", 0), p)
    rng = random.Random("%d %d %d pages" % (batch, case["lo"], case["hi"]))
    free = list(range(n_pages))
    rng.shuffle(free)
    table, refs, lens = [], [0] * n_pages, list(lens)
    for b, n in enumerate(lens):
        if kind == "compact" and b % 2:
            lens[b] = n = 0  # gone
        row = [free.pop() for _ in range(_pages(n, p))]
        if kind == "step" and b % 4 == 1 and lens[b - 1] > p:  # the second of a group shares the first's pages, its last one too
            row, lens[b] = list(table[b - 1]), lens[b - 1]
            row = [x for x in row if x >= 0]
        for x in row:
            refs[x] += 1
        table.append(row + [-1] * (width - len(row)))
    s.update(table=_ints(table, torch.int32), lengths=_ints(lens), refs=_ints(refs, torch.int32),
             table_out=torch.empty(batch, width, dtype=torch.int32, device=DEV),
             refs_out=torch.empty(n_pages, dtype=torch.int32, device=DEV),
             n_pairs=torch.zeros(1, dtype=torch.int32, device=DEV))
    if kind == "step":
        new = _offsets(_new(case))
        s.update(source=_ints(_source(case), torch.int32), new_offsets=_ints(new),
                 rows=torch.empty(new[-1], dtype=torch.int64, device=DEV),
                 lengths_out=torch.empty(batch, dtype=torch.int64, device=DEV),
                 pairs=torch.full((batch, 2), -1, dtype=torch.int32, device=DEV))
    else:
        s["pairs"] = torch.full((n_pages // 2, 2), -1, dtype=torch.int32, device=DEV)
    # keys and values of all layers: [2 layers, rows, kv heads, 128]
    s["caches"] = torch.randn(2 * case["layers"], n_pages * p, case["kv_heads"], D, generator=gen, device=DEV,
                              dtype=torch.bfloat16)
    if own:
        from paper_2607_15621_gb300 import fsx
        s["planes"] = fsx.page_planes(p, caches=list(s["caches"]))
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _answer(s):
    """The outputs of a pass where they are the state's own buffers."""
    kind = s["case"]["kind"]
    if kind == "rotary":
        return [s["q_out"], s["k_out"]] + s["cache"] + s["scale"]
    if kind == "step":
        return [s["table_out"], s["lengths_out"], s["refs_out"], s["rows"], s["pairs"], s["n_pairs"], s["caches"]]
    if kind == "compact":
        return [s["table_out"], s["refs_out"], s["pairs"], s["n_pairs"], s["caches"]]
    if kind == "bounds":
        return [s["bounds"], s["bound_scale"]]
    if kind == "sparse":
        return [s["bounds"], s["bound_scale"], s["picked"], s["out"]]
    return [s["out"], s["lse"]]


def _run_own(s):
    from paper_2607_15621_gb300 import fsx
    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        write = dict(v=s["v"], rows=s["rows"], k_cache=s["cache"][0], v_cache=s["cache"][1], k_scale=s["scale"][0],
                     v_scale=s["scale"][1]) if case["cache"] else {}
        fsx.rotary(s["q"], s["k"], s["positions"], s["pairs"], s["status"], q_out=s["q_out"], k_out=s["k_out"], **write)
    elif kind == "step":
        fsx.pages_step(s["table"], s["lengths"], s["refs"], s["new_offsets"], case["page_rows"], s["table_out"],
                       s["lengths_out"], s["refs_out"], s["rows"], s["pairs"], s["n_pairs"], s["status"], source=s["source"])
        fsx.pages_copy(s["planes"], s["pairs"], s["n_pairs"], s["status"])
    elif kind == "compact":
        fsx.pages_compact(s["table"], s["lengths"], s["refs"], case["page_rows"], s["table_out"], s["refs_out"], s["pairs"],
                          s["n_pairs"], s["status"])
        fsx.pages_copy(s["planes"], s["pairs"], s["n_pairs"], s["status"])
    elif kind == "bounds":
        fsx.page_bounds(s["k_cache"], s["table"], s["lengths"], case["page_rows"], s["bounds"], s["bound_scale"], s["status"],
                        k_scale=s["k_scale"])
    else:
        if kind == "sparse":
            fsx.page_bounds(s["k_cache"], s["table"], s["lengths"], case["page_rows"], s["bounds"], s["bound_scale"],
                            s["status"], k_scale=s["k_scale"], start=s["newest"])
            fsx.page_select(s["q"], s["bounds"], s["bound_scale"], s["table"], s["lengths"], case["page_rows"], s["picked"],
                            s["status"], first=1, last=1)
        fsx.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], case["page_rows"], s["out"],
                            s["status"], s["workspace"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                            picked=s.get("picked"), lse=s["lse"])
    return _answer(s)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "rotary":
        _plain_rotary(s)
    elif kind == "step":
        _plain_step(s)
    elif kind == "compact":
        _plain_compact(s)
    elif kind == "bounds":
        codes, scale = _bounds_of(s, torch.zeros_like(s["lengths"]))
        s["bounds"].copy_(codes)
        s["bound_scale"].copy_(scale)
    else:
        rows, there = _all_rows(s)
        if kind == "sparse":
            codes, scale = _bounds_of(s, s["newest"])
            s["bounds"].copy_(codes)
            s["bound_scale"].copy_(scale)
            s["picked"].copy_(_picked_of(s))
            rows, there = _picked_rows(s)
        o, lse = _attend(s, rows, there)
        s["out"].copy_(o)
        if s["lse"] is not None:
            s["lse"].copy_(lse.T)
    return _answer(s)


def _turn(x, c, z, adjacent):
    """x [rows, heads, 128] with pair j turned: c, z [rows, 64] its cosine and sine."""
    c, z = c[:, None], z[:, None]
    if adjacent:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * z, a * z + b * c], -1).flatten(-2)
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * c - b * z, a * z + b * c], -1)


def _plain_rotary(s):
    case = s["case"]
    angle = s["positions"][s["axis"]].T.double() * s["rate"]  # [rows, 64]; 32 bits would lose far positions
    c, z = torch.cos(angle).float(), torch.sin(angle).float()
    s["q_out"].copy_(_turn(s["q"].float(), c, z, case["adjacent"]))
    k = _turn(s["k"].float(), c, z, case["adjacent"]).to(s["k"].dtype)
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
    if case["cache"] == "e4m3":
        for i, x in enumerate((k, s["v"])):
            code, scale = _codes(x.float())
            s["cache"][i].view(torch.uint8)[s["rows"]] = code.view(torch.uint8)
            s["scale"][i][:, s["rows"]] = scale.T
    elif case["cache"]:
        s["cache"][0][s["rows"]] = k
        s["cache"][1][s["rows"]] = s["v"]


def _all_rows(s):
    """Cache row of every row of every request [batch, 1, most], and which there are."""
    p = s["case"]["page_rows"]
    j = torch.arange(s["most"], device=DEV)
    there = j < s["lengths"][:, None]
    page = s["table"].long()[:, j // p]
    return torch.where(there, page * p + j % p, 0)[:, None], there[:, None]


def _picked_rows(s):
    """The same of the picked pages [batch, kv heads, picked * page_rows]."""
    p = s["case"]["page_rows"]
    logical = s["picked"].long()
    row = logical[..., None] * p + torch.arange(p, device=DEV)
    there = (logical >= 0)[..., None] & (row < s["lengths"][:, None, None, None])
    page = torch.gather(s["table"].long(), 1, logical.clamp(min=0).flatten(1)).view(logical.shape)
    return (torch.where(there, page[..., None] * p + torch.arange(p, device=DEV), 0).flatten(2), there.flatten(2))


def _values(cache, scale, rows):
    """Rows [batch, 1 or kv heads, n] of a cache as [batch, kv heads, n, 128] in 32 bits."""
    head = torch.arange(cache.shape[1], device=DEV)[None, :, None]
    if scale is None:
        return cache[rows, head].float()
    return cache.view(torch.uint8)[rows, head].view(torch.float8_e4m3fn).float() * scale[head, rows][..., None]


def _attend(s, rows, there):
    """Outputs [batch, heads, 128] and log-sum-exps [batch, heads] in 32 bits."""
    b, h, _ = s["q"].shape
    hk = s["k_cache"].shape[1]
    q = s["q"].float().view(b, hk, h // hk, D)
    scores = torch.matmul(q, _values(s["k_cache"], s["k_scale"], rows).transpose(2, 3)) * (1 / math.sqrt(D))
    scores = scores.masked_fill(~there[:, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    v = torch.where(there[..., None], _values(s["v_cache"], s["v_scale"], rows), 0.0)
    o = torch.where(total > 0, torch.matmul(w, v) / total, 0.0)
    return o.view(b, h, D), (top + torch.log(total)).view(b, h)


def _bounds_of(s, start):
    """Codes and scales of all pages: those of the requests' pages from row `start` on made anew, the others as they are."""
    case, hk = s["case"], s["case"]["kv_heads"]
    p, n_pages = case["page_rows"], s["bounds"].shape[0]
    j = torch.arange(s["table"].shape[1], device=DEV)
    mine = (j >= (start // p)[:, None]) & (j * p < s["lengths"][:, None])
    page = s["table"].long()[mine]
    filled = (s["lengths"][:, None] - j * p).clamp(max=p)[mine]
    k = s["k_cache"].view(n_pages, p, hk, D)
    if s["k_scale"] is None:
        k = k[page].float()
    else:
        k = k.view(torch.uint8)[page].view(torch.float8_e4m3fn).float()
        k = k * s["k_scale"].view(hk, n_pages, p)[:, page].permute(1, 2, 0)[..., None]
    there = (torch.arange(p, device=DEV) < filled[:, None])[:, :, None, None]
    lo, hi = torch.where(there, k, math.inf).amin(1), torch.where(there, k, -math.inf).amax(1)
    scale = _least_power(torch.maximum(lo.abs(), hi.abs()).amax(-1), 127)  # [pages, kv heads]
    codes = torch.stack([torch.floor(lo / scale[..., None]), torch.ceil(hi / scale[..., None])], 2)
    bounds, bound_scale = s["bounds"].clone(), s["bound_scale"].clone()
    bounds[page] = codes.to(torch.int8)
    bound_scale[:, page] = scale.T
    return bounds, bound_scale


def _picked_of(s):
    """Logical pages [batch, kv heads, picked], ascending, -1 behind them."""
    case = s["case"]
    b, h, _ = s["q"].shape
    hk, p, most = case["kv_heads"], case["page_rows"], case["picked"]
    q = s["q"].float()
    scale = _least_power(q.abs().amax(-1), 127)
    code = torch.round(q / scale[..., None]).view(b, hk, h // hk, D)
    n = _pages(s["lengths"], p)[:, None]
    width = s["table"].shape[1]
    j = torch.arange(width, device=DEV)
    there = j < n
    page = torch.where(there, s["table"].long(), 0)
    bound = s["bounds"][page].float()  # [batch, width, kv heads, 2, 128]
    lo, hi = bound[:, :, :, 0].permute(0, 2, 3, 1), bound[:, :, :, 1].permute(0, 2, 3, 1)
    total = torch.matmul(code.clamp(min=0), hi) + torch.matmul(code.clamp(max=0), lo)  # whole numbers below 2^22
    power = torch.log2(scale).view(b, hk, -1, 1) + torch.log2(s["bound_scale"][:, page]).permute(1, 0, 2)[:, :, None]
    score = (total * _power(power.round().clamp(-100, 100).int())).amax(2)  # [batch, kv heads, width]
    always = (j < 1) | (j >= n - 1)
    score = torch.where(always[:, None], math.inf, score)
    score = torch.where(there[:, None], score, -math.inf)
    rank = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :most]  # ties: the lowest page first
    if rank.shape[-1] < most:
        rank = torch.nn.functional.pad(rank, (0, most - rank.shape[-1]), value=width)
    rank = torch.where(rank < n[:, None], rank, width + 1)
    rank = torch.sort(rank, dim=-1)[0]
    return torch.where(rank > width, -1, rank).to(torch.int32)


def _count(n, at, mask, by):
    """How often each of 0 .. n - 1 is named by `at` where `mask`, times `by`."""
    got = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
    got.index_add_(0, torch.where(mask, at.long(), n).flatten(), torch.full((at.numel(),), by, device=DEV))
    return got[:n]


def _plain_step(s):
    table, lengths, p = s["table"], s["lengths"], s["case"]["page_rows"]
    batch, width = table.shape
    n_pages = s["refs"].shape[0]
    j, i = torch.arange(width, device=DEV), torch.arange(batch, device=DEV)
    src = s["source"].long()
    n = torch.where(src >= 0, lengths[src.clamp(min=0)], 0)
    add = s["new_offsets"][1:] - s["new_offsets"][:-1]
    mine = table[src.clamp(min=0)]
    had = _pages(n, p)
    refs = (s["refs"].long() + _count(n_pages, table, j * p < lengths[:, None], -1)
            + _count(n_pages, mine, j < had[:, None], 1))
    # the last page, where new tokens go into it: a request that shares it copies it, but for the last one if nobody else holds it
    last = torch.gather(mine, 1, (had - 1).clamp(min=0)[:, None])[:, 0].long()
    into = (n % p > 0) & (add > 0)
    held, writers = refs[last], _count(n_pages, last, into, 1)[last]
    behind = torch.zeros(n_pages + 1, dtype=torch.int64, device=DEV).scatter_reduce_(
        0, torch.where(into, last, n_pages), i, "amax", include_self=False)[last]
    copies = into & (held > 1) & ~((held == writers) & (i == behind))
    kept = had - copies.long()
    need = torch.where(add > 0, _pages(n + add, p) - kept, 0)
    end = need.cumsum(0)
    grows = (end <= (refs == 0).sum()) | (need == 0)
    copies, need_now = copies & grows, torch.where(grows, need, 0)
    free = torch.sort((refs > 0).int(), stable=True)[1]  # the free pages first, lowest first
    kept = torch.where(grows, kept, had)
    fresh = (j >= kept[:, None]) & (j < (kept + need_now)[:, None])
    page = free[((end - need)[:, None] + j - kept[:, None]).clamp(0, n_pages - 1)]
    out = torch.where(j < kept[:, None], mine.long(), torch.where(fresh, page, -1))
    refs = refs - _count(n_pages, last, copies, 1) + _count(n_pages, out, fresh, 1)
    s["table_out"].copy_(out)
    s["refs_out"].copy_(refs)
    s["lengths_out"].copy_(n + torch.where(grows, add, 0))
    t = torch.arange(s["rows"].shape[0], device=DEV)
    b = torch.searchsorted(s["new_offsets"][1:], t, right=True)
    at = n[b] + t - s["new_offsets"][b]
    s["rows"].copy_(torch.where(grows[b], out[b, at // p] * p + at % p, -1))
    to = torch.where(copies, copies.long().cumsum(0) - 1, batch)
    pairs = torch.cat([s["pairs"].long(), torch.zeros(1, 2, dtype=torch.int64, device=DEV)])
    pairs[to] = torch.stack([last, torch.gather(out, 1, (had - 1).clamp(min=0)[:, None])[:, 0]], 1)
    s["pairs"].copy_(pairs[:batch])
    s["n_pairs"].copy_(copies.sum())
    _plain_copy(s)


def _plain_compact(s):
    refs, p = s["refs"].long(), s["case"]["page_rows"]
    n_pages, most = refs.shape[0], s["pairs"].shape[0]
    i = torch.arange(n_pages, device=DEV)
    used = refs > 0
    first = used.sum()
    moves, room = used & (i >= first), ~used & (i < first)
    pairs = torch.cat([s["pairs"].long(), torch.zeros(1, 2, dtype=torch.int64, device=DEV)])
    pairs[torch.where(moves, moves.long().cumsum(0) - 1, most), 0] = i
    pairs[torch.where(room, room.long().cumsum(0) - 1, most), 1] = i
    s["pairs"].copy_(pairs[:most])
    s["n_pairs"].copy_(moves.sum())
    to = torch.where(moves, pairs[torch.where(moves, moves.long().cumsum(0) - 1, most), 1], i)
    table = s["table"].long()
    mine = torch.arange(table.shape[1], device=DEV) * p < s["lengths"][:, None]
    s["table_out"].copy_(torch.where(mine, to[table.clamp(min=0)], table))
    s["refs_out"].copy_(torch.zeros(n_pages, dtype=torch.int64, device=DEV).index_add_(0, to, refs))
    _plain_copy(s)


def _plain_copy(s):
    pairs = s["pairs"][:int(s["n_pairs"])].long()
    pages = s["caches"].view(s["caches"].shape[0], s["refs"].shape[0], -1)
    pages[:, pairs[:, 1]] = pages[:, pairs[:, 0]]


def _copied(case):
    """step: pages that are copied, by the case alone: of the requests that write into a shared last page all but the last."""
    src, new = _source(case), _new(case)
    lens, p = _lengths(case), case["page_rows"]
    for b in range(1, len(lens), 4):
        if lens[b - 1] > p:
            lens[b] = lens[b - 1]
    shared = {}
    for b, a in enumerate(src):
        if a >= 0 and lens[a] % p:
            shared.setdefault(a - 1 if a % 4 == 1 and lens[a - 1] > p else a, []).append(b)
    return sum(len(v) - 1 for v in shared.values())


def work(case):
    kind, hk = case["kind"], case["kv_heads"]
    if kind == "rotary":
        n, h, size = case["rows"], case["heads"], SIZE[case["dtype"]]
        move = 2 * n * h * D * size + n * hk * D * size + 8 * n * case["axes"]
        if case["keys"]:
            move += n * hk * D * size
        if case["cache"]:
            move += n * hk * D * size + 2 * n * hk * (D * SIZE[case["cache"]] + (4 if case["cache"] == "e4m3" else 0)) + 8 * n
        return {"bytes": move, "flops": 3 * n * (h + hk) * D}
    lens, p = _lengths(case), case["page_rows"]
    if kind in ("step", "compact"):
        page = 2 * 2 * case["layers"] * 2 * p * hk * D  # in and out
        entries = 4 * sum(_pages(n, p) for n in lens)
        if kind == "step":
            return {"bytes": 2 * entries + 8 * case["pages"] + 8 * sum(_new(case)) + 32 * case["batch"] + _copied(case) * page, "flops": 0}
        used = sum(_pages(n, p) for n in lens[::2])
        moved = round(used * (1 - used / case["pages"]))  # as many as lie behind the first `used` pages, on average
        return {"bytes": entries + 8 * case["pages"] + moved * page, "flops": 0}
    row = D * SIZE[case["cache"]] + (4 if case["cache"] == "e4m3" else 0)
    pages = sum(_pages(n, p) for n in lens)
    if kind == "bounds":
        return {"bytes": sum(lens) * hk * row + pages * (hk * (2 * D + 4) + 4), "flops": 2 * sum(lens) * hk * D}
    b, h = case["batch"], case["heads"]
    move = 2 * b * h * D * SIZE[case["dtype"]] + (4 * b * h if case.get("lse") else 0)
    if kind == "paged":
        return {"bytes": move + 2 * sum(lens) * hk * row + 4 * pages, "flops": 4 * D * h * sum(lens)}
    took = sum(min(n, case["picked"] * p) for n in lens)
    newest = sum(min(n, (n - 1) % p + 1) for n in lens if n)
    move += pages * (hk * (2 * D + 4) + 4) + newest * hk * row + 2 * took * hk * row + b * hk * (4 * case["picked"] + 2 * D + 4)
    return {"bytes": move, "flops": 2 * 2 * D * h * pages + 4 * D * h * took}


def _cache64(s, x, rows, head):
    """Rows of one kv head of a cache in 64 bits."""
    c = s[x + "_cache"][:, head]
    if s[x + "_scale"] is None:
        return c[rows].double()
    return c.view(torch.uint8)[rows].view(torch.float8_e4m3fn).double() * s[x + "_scale"][head, rows].double()[:, None]


def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _power64(top, most):
    """The smallest power of two >= 2^-126 that brings `top` to `most` or below, by its logarithm and two looks."""
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / most)) - 1
    e = torch.where(top > most * _two(e), e + 1, e)
    e = torch.where(top > most * _two(e), e + 1, e).clamp(min=-126)
    return torch.where(top > 0, _two(e), torch.ones_like(top))


def _exact_rotary(s, case):
    _, axis, rate = _pairs(case)
    where = torch.stack([s["positions"][a].double() * r for a, r in zip(axis, rate)], 1)
    turn = torch.polar(torch.ones_like(where), where)[:, None]

    def turned(x):
        x = x.double()
        z = torch.view_as_complex(x.unflatten(-1, (64, 2)) if case["adjacent"] else torch.stack([x[..., :64], x[..., 64:]], -1).contiguous()) * turn
        return torch.view_as_real(z).flatten(-2) if case["adjacent"] else torch.cat([z.real, z.imag], -1)

    q, k = turned(s["q"]), turned(s["k"])
    out = [q, k if case["keys"] else None]
    rounded = k.to(s["k"].dtype).double()  # keys are stored from what they are in the operator's type
    if case["cache"] is None:
        return out
    caches, scales = [], []
    for x, c in zip((rounded if case["cache"] == "e4m3" else k, s["v"].double()), s["cache"]):
        whole = torch.zeros(c.shape, dtype=torch.float64, device=DEV)
        if case["cache"] == "e4m3":
            top = x.abs().amax(-1)
            scale = _power64(top, 448.0)
            y = x / scale[..., None]
            step = _two(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)  # 3 bits behind the leading one
            x = torch.round(y / step) * step
            z = torch.ones(c.shape[1], c.shape[0], dtype=torch.float64, device=DEV)
            z[:, s["rows"]] = scale.T
            scales.append(z)
        whole[s["rows"]] = x
        caches.append(whole)
    return out + caches + scales


def _exact_bounds(s, case, start):
    """Page by page of each request; the others as they are."""
    p, hk = case["page_rows"], case["kv_heads"]
    bounds, scale = s["bounds"].clone(), s["bound_scale"].double()
    table = s["table"].tolist()
    for b, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        first = start[b] // p
        pages = _ints(table[b][first:_pages(n, p)])
        rows = (pages[:, None] * p + torch.arange(p, device=DEV)).flatten()
        k = torch.stack([_cache64(s, "k", rows, h) for h in range(hk)], 1).view(-1, p, hk, D)
        spare = len(pages) * p - (n - first * p)
        if spare:  # rows behind the request: the first row of the page in their place
            k[-1, p - spare:] = k[-1, :1]
        z = _power64(k.abs().amax((1, 3)), 127.0)
        bounds[pages, :, 0] = torch.floor(k.amin(1) / z[..., None]).to(torch.int8)
        bounds[pages, :, 1] = torch.ceil(k.amax(1) / z[..., None]).to(torch.int8)
        scale[:, pages] = z.T
    return bounds, scale


def _exact_picked(s, case, bounds, scale):
    p, hk, most = case["page_rows"], case["kv_heads"], case["picked"]
    b, h = case["batch"], case["heads"]
    q = s["q"].double()
    z = _power64(q.abs().amax(-1), 127.0)
    code = torch.round(q / z[..., None]).cpu()
    got = torch.full((b, hk, most), -1, dtype=torch.int32)
    z, bounds, scale, table = z.cpu(), bounds.cpu().double(), scale.cpu(), s["table"].tolist()
    for i, n in enumerate(s["lengths"].tolist()):
        pages = table[i][:_pages(n, p)]
        for head in range(hk):
            best = None
            for c, w in zip(code[i, head * (h // hk):(head + 1) * (h // hk)], z[i, head * (h // hk):(head + 1) * (h // hk)]):
                up = torch.maximum(bounds[pages, head, 0] * c, bounds[pages, head, 1] * c).sum(1) * w * scale[head, pages]
                best = up if best is None else torch.maximum(best, up)
            best = best.tolist()
            rest = sorted(range(1, len(pages) - 1), key=lambda x: (-best[x], x))[:max(0, most - 2)]
            took = sorted(rest + list({0, len(pages) - 1} if pages else ()))
            got[i, head, :len(took)] = torch.tensor(took, dtype=torch.int32)
    return got.to(DEV)


def _exact_step(s, case):
    """Request by request, with lists."""
    p, table, lens, refs = case["page_rows"], s["table"].tolist(), s["lengths"].tolist(), s["refs"].tolist()
    new = _new(case)
    held = [table[a][:_pages(lens[a], p)] if a >= 0 else [] for a in _source(case)]
    n = [lens[a] if a >= 0 else 0 for a in _source(case)]
    for b, row in enumerate(table):
        for x in row[:_pages(lens[b], p)]:
            refs[x] -= 1
    for row in held:
        for x in row:
            refs[x] += 1
    free = [x for x, r in enumerate(refs) if r == 0]
    moved, rows, left = [], [], dict(enumerate(refs))
    for b, add in enumerate(new):
        row = held[b]
        if add and n[b] % p and left[row[-1]] > 1:
            left[row[-1]] -= 1
            left[free[0]] = 1
            moved.append([row[-1], free[0]])
            row = row[:-1] + [free.pop(0)]
        while len(row) * p < n[b] + add:
            left[free[0]] = 1
            row = row + [free.pop(0)]
        held[b] = row
        rows += [row[x // p] * p + x % p for x in range(n[b], n[b] + add)]
    caches = s["caches"].double()
    pages = caches.view(caches.shape[0], len(refs), -1)
    for a, c in moved:
        pages[:, c] = pages[:, a]
    width = s["table"].shape[1]
    pairs = s["pairs"].clone()
    pairs[:len(moved)] = _ints(moved, torch.int32).view(-1, 2)
    return [_ints([r + [-1] * (width - len(r)) for r in held], torch.int32), _ints([x + y for x, y in zip(n, new)]),
            _ints([left[x] for x in range(len(refs))], torch.int32), _ints(rows), pairs, _ints([len(moved)], torch.int32), caches]


def _exact_compact(s, case):
    p, refs, table = case["page_rows"], s["refs"].tolist(), s["table"].tolist()
    used = [x for x, r in enumerate(refs) if r > 0]
    moved = list(zip([x for x in used if x >= len(used)], [x for x, r in enumerate(refs[:len(used)]) if r <= 0]))
    to = dict(moved)
    caches = s["caches"].double()
    pages = caches.view(caches.shape[0], len(refs), -1)
    for a, c in moved:
        pages[:, c] = pages[:, a]
        refs[a], refs[c] = 0, refs[a]
    for row, n in zip(table, s["lengths"].tolist()):
        for x in range(_pages(n, p)):
            row[x] = to.get(row[x], row[x])
    pairs = s["pairs"].clone()
    pairs[:len(moved)] = _ints(moved, torch.int32).view(-1, 2)
    return [_ints(table, torch.int32), _ints(refs, torch.int32), pairs, _ints([len(moved)], torch.int32), caches]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        return _exact_rotary(s, case)
    if kind == "step":
        return _exact_step(s, case)
    if kind == "compact":
        return _exact_compact(s, case)
    if kind == "bounds":
        return list(_exact_bounds(s, case, [0] * case["batch"]))
    p, hk, g = case["page_rows"], case["kv_heads"], case["heads"] // case["kv_heads"]
    picked = None
    if kind == "sparse":
        bounds, scale = _exact_bounds(s, case, s["newest"].tolist())
        picked = _exact_picked(s, case, bounds, scale)
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full((case["heads"], case["batch"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        at = torch.arange(n, device=DEV)
        row = s["table"][b].long()[at // p] * p + at % p
        for head in range(hk):
            rows = row
            if picked is not None:
                rows = row[torch.isin(at // p, picked[b, head].long())]
            a = s["q"][b, head * g:(head + 1) * g].double() @ _cache64(s, "k", rows, head).T / math.sqrt(D)
            z = torch.logsumexp(a, 1)
            o[b, head * g:(head + 1) * g] = torch.exp(a - z[:, None]) @ _cache64(s, "v", rows, head)
            lse[head * g:(head + 1) * g, b] = z
    return [bounds, scale, picked, o] if kind == "sparse" else [o, lse if case["lse"] else None]
