"""The language-model operators next to the tick and the append, as cases whose time and results can be measured.

Kinds of call (field "kind"):
  prompt  attention over whole prompts, packed one after another, causal or not, with grouped heads (prompt_attention)
  write   rows of keys and values quantised to 8 bits as they are written into a cache (cache_write)
  read    rows of an 8-bit cache read back as 16- or 32-bit values (cache_read)
  tree    a few drafted tokens of each request over its cache, 16-bit or 8-bit, and over the drafted tokens that a mask
          of theirs lets them see; one token a request is plain decoding (tree_attention)

Shapes are the repository's own: 32 heads of 128 of a 7B-shaped backbone, histories from a few rows (64 instruction
tokens and 40 frames x 4 are 224) to those of its sweep and beyond, one vehicle to a fleet of 128; and the same with
grouped key/value heads. Values follow the synthetic workloads: keys ~ N(0, 1) times a log-normal scale per head and
dimension, queries and values ~ N(0, 1), rounded to the type.

The 8-bit cache: e4m3 codes with one scale per row and head, the smallest power of two that brings the row's largest
magnitude to 448 or below. Scales lie as [heads, rows].
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
D = 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}


def listed():
    return [
        # one vehicle's first prompt: 64 instruction tokens + 40 frames x 4; projections in one fused buffer
        dict(name="prompt_b1_224", kind="prompt", batch=1, lo=224, hi=224, past=0, heads=32, kv_heads=32, dtype="bf16",
             causal=True, fused=True, lse=False),
        # a small fleet's prompts, ragged, grouped heads
        dict(name="prompt_b16_ragged", kind="prompt", batch=16, lo=96, hi=480, past=0, heads=32, kv_heads=8,
             dtype="bf16", causal=True, fused=True, lse=False),
        # chunks of new tokens behind rows that are already there, with log-sum-exps for a later merge
        dict(name="prompt_chunk_b4", kind="prompt", batch=4, lo=100, hi=517, past=2048, heads=32, kv_heads=32,
             dtype="fp16", causal=True, fused=False, lse=True),
        # one long history from scratch: the largest case
        dict(name="prompt_b1_8192", kind="prompt", batch=1, lo=8192, hi=8192, past=0, heads=32, kv_heads=8,
             dtype="bf16", causal=True, fused=True, lse=False),
        # one frame's four tokens on their way into the cache: latency
        dict(name="write_frame", kind="write", rows=4, cache_rows=4096, kv_heads=32, dtype="bf16", fused=True),
        # the rows of a fleet's prompts, from 32-bit values
        dict(name="write_fleet", kind="write", rows=28001, cache_rows=65536, kv_heads=32, dtype="fp32", fused=False),
        # a vehicle's history, grouped heads, read back for a 16-bit consumer
        dict(name="read_history", kind="read", rows=517, cache_rows=4096, kv_heads=8, dtype="fp16"),
        # a fleet's rows, read back
        dict(name="read_fleet", kind="read", rows=50000, cache_rows=65536, kv_heads=32, dtype="bf16"),
        # one request decoding a single token over the cache as the append writes it
        dict(name="tree_b1_single", kind="tree", batch=1, lo=224, hi=224, new=1, heads=32, kv_heads=32, dtype="bf16",
             cache="bf16", lse=False),
        # a small fleet verifying drafts of up to 11 tokens over its 8-bit caches, grouped heads
        dict(name="tree_b16_drafts", kind="tree", batch=16, lo=96, hi=480, new=11, heads=32, kv_heads=8, dtype="bf16",
             cache="e4m3", lse=False),
        # one request with a long history and a wide tree
        dict(name="tree_b1_wide_32768", kind="tree", batch=1, lo=32768, hi=32768, new=63, heads=32, kv_heads=8,
             dtype="bf16", cache="e4m3", lse=True),
        # the fleet batch of the benchmark, one token a vehicle, over 8-bit caches
        dict(name="tree_b128_single", kind="tree", batch=128, lo=64, hi=2048, new=1, heads=32, kv_heads=32,
             dtype="bf16", cache="e4m3", lse=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "tree", "tree", "write", "read"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32, 32])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "prompt":
        heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if kv_heads * g <= 32])
        past = rng.choice([0, 0, 1]) * _log(rng, 16, 4096)
        causal = rng.random() < 0.8
        most = (8192 if causal else 5500) - past
        batch = _log(rng, 1, 32)
        hi = _log(rng, 1, max(2, most // batch))
        lo = max(1, _log(rng, max(1, hi // 8), hi))
        return dict(kind=kind, batch=batch, lo=lo, hi=hi, past=past, heads=heads, kv_heads=kv_heads, dtype=dtype,
                    causal=causal, fused=past == 0 and rng.random() < 0.5, lse=rng.random() < 0.3)
    if kind == "tree":
        heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if kv_heads * g <= 32])
        batch = _log(rng, 1, 128)
        hi = _log(rng, 1, min(32768, 131072 // batch))
        lo = max(0, _log(rng, max(1, hi // 16), hi) - 1)
        return dict(kind=kind, batch=batch, lo=lo, hi=hi, new=_log(rng, 1, 64), heads=heads, kv_heads=kv_heads,
                    dtype=dtype, cache=rng.choice(["e4m3", "e4m3", dtype]), lse=rng.random() < 0.3)
    rows = _log(rng, 1, 28000)
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    case = dict(kind=kind, rows=rows, cache_rows=rows + rng.randrange(4, 4096), kv_heads=kv_heads, dtype=dtype)
    if kind == "write":
        case["fused"] = rng.random() < 0.5
    return case


def _lengths(case):
    """Lengths of the case's sequences or caches, and of its drafts: part of the case, not of the seed."""
    rng = random.Random("%d %d %d" % (case["batch"], case["lo"], case["hi"]))
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    past = [rng.randint(case["past"] // 2, case["past"]) for _ in lens] if case.get("past") else [0] * len(lens)
    new = [rng.randint((case["new"] + 1) // 2, case["new"]) for _ in lens] if "new" in case else None
    return lens, past, new


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _keys(gen, rows, heads):
    scale = torch.exp(0.5 * torch.randn(heads, D, generator=gen, device=DEV))
    return torch.randn(rows, heads, D, generator=gen, device=DEV) * scale


def _i64(v):
    return torch.tensor(v, dtype=torch.int64, device=DEV)


def _power(e):
    """2^e in 32 bits, exactly, for -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x):
    """e4m3 codes and scales of rows [..., 128] in 32 bits."""
    top = x.abs().amax(-1)
    e = torch.frexp(top)[1] - 9  # top = f 2^E with f in [1/2, 1): top / 2^(E - 9) lies in [256, 512)
    e = e.clamp(-126, 119)
    e = torch.where(top / _power(e) > 448, e + 1, e)
    scale = torch.where(top > 0, _power(e), torch.ones_like(top))
    return (x / scale[..., None]).to(torch.float8_e4m3fn), scale


def _tree_masks(gen_cpu, new):
    """One 64-bit word per drafted token: itself and its ancestors in a random tree."""
    words = []
    for n in new:
        mine = []
        for i in range(n):
            parent = int(torch.randint(-1, i, (1,), generator=gen_cpu)) if i else -1
            mine.append((mine[parent] if parent >= 0 else 0) | (1 << i))
        words += mine
    return [w - (1 << 64) if w >= 1 << 63 else w for w in words]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    kind, hk = case["kind"], case["kv_heads"]
    t = TYPES[case["dtype"]]
    if kind == "prompt":
        h = case["heads"]
        lens, past, _ = _lengths(case)
        qo, ko = _offsets(lens), _offsets([a + b for a, b in zip(lens, past)])
        q = torch.randn(qo[-1], h, D, generator=gen, device=DEV)
        k, v = _keys(gen, ko[-1], hk), torch.randn(ko[-1], hk, D, generator=gen, device=DEV)
        if case["fused"]:  # q, k, v as the columns of one projection's output
            buf = torch.cat([q, k, v], 1).to(t)
            q, k, v = buf[:, :h], buf[:, h:h + hk], buf[:, h + hk:]
        else:
            q, k, v = q.to(t), k.to(t), v.to(t)
        s.update(q=q, k=k, v=v, q_offsets=_i64(qo), kv_offsets=_i64(ko), most=(max(lens), max(a + b for a, b in zip(lens, past))),
                 out=torch.empty(qo[-1], h, D, dtype=t, device=DEV),
                 lse=torch.empty(h, qo[-1], device=DEV) if case["lse"] else None)
    elif kind in ("write", "read"):
        n, m = case["rows"], case["cache_rows"]
        first = seed % (m - n + 1)
        s["rows"] = torch.arange(first, first + n, dtype=torch.int64, device=DEV)
        k, v = _keys(gen, n, hk), torch.randn(n, hk, D, generator=gen, device=DEV)
        if kind == "write":
            if case["fused"]:
                buf = torch.cat([k, v], 1).to(t)
                s["k"], s["v"] = buf[:, :hk], buf[:, hk:]
            else:
                s["k"], s["v"] = k.to(t), v.to(t)
            s["cache"] = [torch.zeros(m, hk, D, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in "kv"]
            s["scale"] = [torch.ones(hk, m, device=DEV) for _ in "kv"]
        else:
            s["cache"] = [torch.zeros(m, hk, D, dtype=torch.uint8, device=DEV) for _ in "kv"]
            s["scale"] = [torch.ones(hk, m, device=DEV) for _ in "kv"]
            for x, c, z in zip((k, v), s["cache"], s["scale"]):
                code, scale = _codes(x)
                c[first:first + n] = code.view(torch.uint8)
                z[:, first:first + n] = scale.T
            s["cache"] = [c.view(torch.float8_e4m3fn) for c in s["cache"]]
            s["k"], s["v"] = (torch.empty(n, hk, D, dtype=t, device=DEV) for _ in "kv")
    else:
        h = case["heads"]
        lens, _, new = _lengths(case)
        no = _offsets(new)
        gap = case["new"]  # free rows behind every request's cache, where accepted tokens go
        starts = _offsets([n + gap for n in lens])
        rows = starts.pop()
        k, v = _keys(gen, rows, hk), torch.randn(rows, hk, D, generator=gen, device=DEV)
        if case["cache"] == "e4m3":
            (ck, sk), (cv, sv) = _codes(k), _codes(v)
            s["cache"], s["scale"] = [ck, cv], [sk.T.contiguous(), sv.T.contiguous()]
            del sk, sv
        else:
            s["cache"], s["scale"] = [k.to(t), v.to(t)], [None, None]
        del k, v
        buf = torch.cat([torch.randn(no[-1], h, D, generator=gen, device=DEV), _keys(gen, no[-1], hk),
                         torch.randn(no[-1], hk, D, generator=gen, device=DEV)], 1).to(t)
        gen_cpu = torch.Generator().manual_seed(seed)
        s.update(q=buf[:, :h], k=buf[:, h:h + hk], v=buf[:, h + hk:], new_offsets=_i64(no), mask=_i64(_tree_masks(gen_cpu, new)),
                 starts=_i64(starts), offsets=_i64(_offsets(lens)), most=(max(new), max(lens)),
                 out=torch.empty(no[-1], h, D, dtype=t, device=DEV),
                 lse=torch.empty(h, no[-1], device=DEV) if case["lse"] else None)
        if own:
            from paper_2607_15621_gb300 import fsx
            s["workspace"] = torch.zeros(fsx.tree_attention_workspace_bytes(case["batch"], no[-1], h, hk), dtype=torch.uint8, device=DEV)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2607_15621_gb300 import fsx
    kind = s["case"]["kind"]
    if kind == "prompt":
        fsx.prompt_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["kv_offsets"], s["out"], s["status"], lse=s["lse"],
                             causal=s["case"]["causal"])
    elif kind == "write":
        fsx.cache_write(s["k"], s["v"], s["rows"], *s["cache"], *s["scale"], s["status"])
        return s["cache"] + s["scale"]
    elif kind == "read":
        fsx.cache_read(*s["cache"], *s["scale"], s["rows"], s["k"], s["v"], s["status"])
        return [s["k"], s["v"]]
    else:
        fsx.tree_attention(s["q"], s["k"], s["v"], s["new_offsets"], s["mask"], *s["cache"], s["offsets"], s["out"],
                           s["status"], s["workspace"], k_scale=s["scale"][0], v_scale=s["scale"][1], starts=s["starts"],
                           lse=s["lse"])
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


def _padded(x, start, lens, most):
    """Rows start[b] .. start[b] + lens[b] - 1 of x as [batch, most, ...] in 32 bits, zeros behind them; and which are rows."""
    i = torch.arange(most, device=DEV)
    there = i < lens[:, None]
    at = torch.where(there, start[:, None] + i, 0)
    got = x[at].float()
    return torch.where(there.view(there.shape + (1,) * (x.dim() - 1)), got, 0.0), there


def _softmax_v(q, k, v, see):
    """q [b, t, heads, 128], k and v [b, n, kv heads, 128], see [b, t, n]: outputs [b, t, heads, 128], lse [b, t, heads]."""
    b, t, h, _ = q.shape
    hk, n = k.shape[2], k.shape[1]
    g = h // hk
    q = q.view(b, t, hk, g, D).permute(0, 2, 3, 1, 4).reshape(b, hk, g * t, D)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1)) * (1 / math.sqrt(D))
    scores = scores.view(b, hk, g, t, n).masked_fill_(~see[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, g * t, n), v.transpose(1, 2)).view(b, hk, g, t, D)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (top + torch.log(total)).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(b, t, h, D), lse.permute(0, 3, 1, 2).reshape(b, t, h)


def _packed(x, offsets, rows):
    """Row i of a packed tensor out of [batch, most, ...]."""
    i = torch.arange(rows, device=DEV)
    b = torch.searchsorted(offsets[1:], i, right=True)
    return x[b, i - offsets[b]]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "prompt":
        qo, ko = s["q_offsets"], s["kv_offsets"]
        nq, nk = qo[1:] - qo[:-1], ko[1:] - ko[:-1]
        q, _ = _padded(s["q"], qo[:-1], nq, s["most"][0])
        k, there = _padded(s["k"], ko[:-1], nk, s["most"][1])
        v, _ = _padded(s["v"], ko[:-1], nk, s["most"][1])
        see = there[:, None, :].expand(-1, q.shape[1], -1)
        if case["causal"]:
            i, j = torch.arange(q.shape[1], device=DEV), torch.arange(k.shape[1], device=DEV)
            see = see & (j <= i[:, None] + (nk - nq)[:, None, None])
        o, lse = _softmax_v(q, k, v, see)
        o, lse = _packed(o, qo, s["q"].shape[0]), _packed(lse, qo, s["q"].shape[0])
    elif kind == "write":
        for x, c, z in zip((s["k"], s["v"]), s["cache"], s["scale"]):
            code, scale = _codes(x.float())
            c.view(torch.uint8)[s["rows"]] = code.view(torch.uint8)
            z[:, s["rows"]] = scale.T
        return s["cache"] + s["scale"]
    elif kind == "read":
        return [(c.view(torch.uint8)[s["rows"]].view(torch.float8_e4m3fn).float() * z[:, s["rows"]].T[..., None]).to(s["k"].dtype)
                for c, z in zip(s["cache"], s["scale"])]
    else:
        no = s["new_offsets"]
        nn, lens = no[1:] - no[:-1], s["offsets"][1:] - s["offsets"][:-1]
        q, _ = _padded(s["q"], no[:-1], nn, s["most"][0])
        kn, is_new = _padded(s["k"], no[:-1], nn, s["most"][0])
        vn, _ = _padded(s["v"], no[:-1], nn, s["most"][0])
        cached = []
        for c, z in zip(s["cache"], s["scale"]):
            if z is None:
                x, there = _padded(c, s["starts"], lens, s["most"][1])
            else:
                x, there = _padded(c.view(torch.uint8), s["starts"], lens, s["most"][1])
                x = x.to(torch.uint8).view(torch.float8_e4m3fn).float() * _padded(z.T, s["starts"], lens, s["most"][1])[0][..., None]
            cached.append(x)
        words, _ = _padded(s["mask"].view(-1, 1) >> torch.arange(s["most"][0], device=DEV) & 1, no[:-1], nn, s["most"][0])
        see = torch.cat([there[:, None, :].expand(-1, q.shape[1], -1), (words > 0) & is_new[:, None, :]], 2)
        o, lse = _softmax_v(q, torch.cat([cached[0], kn], 1), torch.cat([cached[1], vn], 1), see)
        o, lse = _packed(o, no, s["q"].shape[0]), _packed(lse, no, s["q"].shape[0])
    o = o.to(s["out"].dtype)
    return [o] if s["lse"] is None else [o, lse.T.contiguous()]


def work(case):
    kind, hk = case["kind"], case["kv_heads"]
    if kind in ("write", "read"):
        n = case["rows"]
        return {"bytes": 2 * n * hk * (D * (SIZE[case["dtype"]] + 1) + 4) + 8 * n, "flops": 2 * n * hk * D * 2}
    h = case["heads"]
    lens, past, new = _lengths(case)
    size = SIZE[case["dtype"]]
    if kind == "prompt":
        pairs = sum(n * p + (n * (n + 1) // 2 if case["causal"] else n * n) for n, p in zip(lens, past))
        move = 2 * sum(lens) * h * D * size + 2 * (sum(lens) + sum(past)) * hk * D * size
        rows = sum(lens)
    else:
        pairs = sum(t * n + (t * (t + 1) // 2 if t > 1 else 1) for n, t in zip(lens, new))
        row = D * SIZE[case["cache"]] + (4 if case["cache"] == "e4m3" else 0)
        rows = sum(new)
        move = 2 * sum(lens) * hk * row + 2 * rows * (h + hk) * D * size + 8 * rows
    return {"bytes": move + (4 * rows * h if case["lse"] else 0), "flops": 4 * D * h * pairs}


def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """Codes as values and scales of rows in 64 bits: the nearest multiple of the e4m3 step at each magnitude, ties to even."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 448)) - 1
    e = torch.where(top > 448 * _power64(e), e + 1, e)
    e = torch.where(top > 448 * _power64(e), e + 1, e).clamp(min=-126)
    scale = torch.where(top > 0, _power64(e), torch.ones_like(top))
    y = x / scale
    step = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)  # 3 bits behind the leading one
    return torch.round(y / step) * step, scale[..., 0]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "write":
        out = []
        for x, c in zip((s["k"], s["v"]), s["cache"]):
            code, scale = _exact_rows(x.double())
            whole = torch.zeros(c.shape, dtype=torch.float64, device=DEV)
            whole[s["rows"]] = code
            z = torch.ones(c.shape[1], c.shape[0], dtype=torch.float64, device=DEV)
            z[:, s["rows"]] = scale.T
            out.append((whole, z))
        return [out[0][0], out[1][0], out[0][1], out[1][1]]
    if kind == "read":
        at = int(s["rows"][0])
        return [c[at:at + case["rows"]].double() * z[:, at:at + case["rows"]].T.double()[..., None] for c, z in zip(s["cache"], s["scale"])]
    h, g = case["heads"], case["heads"] // case["kv_heads"]
    o = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(h, o.shape[0], dtype=torch.float64, device=DEV)
    lens, past, new = _lengths(case)
    q_at = _offsets(lens if kind == "prompt" else new)
    for b, n in enumerate(lens):
        q = s["q"][q_at[b]:q_at[b + 1]].double()
        if kind == "prompt":
            k0 = int(s["kv_offsets"][b])
            k, v = (s[x][k0:k0 + n + past[b]].double() for x in "kv")
            see = torch.ones(n, n + past[b], dtype=torch.bool, device=DEV)
            see = see.tril(past[b]) if case["causal"] else see
        else:
            r0, t = int(s["starts"][b]), new[b]
            k, v = (c[r0:r0 + n].double() for c in s["cache"])
            if case["cache"] == "e4m3":
                k, v = (x * z[:, r0:r0 + n].T.double()[..., None] for x, z in zip((k, v), s["scale"]))
            k, v = (torch.cat([x, s[y][q_at[b]:q_at[b + 1]].double()]) for x, y in zip((k, v), "kv"))
            bits = [[w >> j & 1 for j in range(t)] for w in s["mask"][q_at[b]:q_at[b + 1]].tolist()]
            see = torch.cat([torch.ones(t, n, dtype=torch.bool, device=DEV), torch.tensor(bits, device=DEV) > 0], 1)
        for head in range(h):
            a = q[:, head] @ k[:, head // g].T / math.sqrt(D) + torch.where(see, 0.0, -math.inf)
            z = torch.logsumexp(a, 1)
            o[q_at[b]:q_at[b + 1], head] = torch.exp(a - z[:, None]) @ v[:, head // g]
            lse[head, q_at[b]:q_at[b + 1]] = z
    return [o] if s["lse"] is None else [o, lse]
