"""Definitions in 64 bits and in lists of the operators over a cache in pages (numpy only).

Every function follows its definition row by row or request by request; nothing is shared with the library.
"""
from __future__ import annotations

import math

import numpy as np

from .llm_oracle import attention_row


def rotary(x, positions, axis, rate, adjacent=False):
    """x [rows, heads, 128], positions [axes, rows]: pair j turned by positions[axis[j]] * rate[j] radians."""
    out = np.array(x, dtype=np.float64)
    for r in range(x.shape[0]):
        for j in range(64):
            a, b = (2 * j, 2 * j + 1) if adjacent else (j, j + 64)
            t = float(positions[axis[j], r]) * rate[j]
            c, s = math.cos(t), math.sin(t)
            out[r, :, a] = x[r, :, a] * c - x[r, :, b] * s
            out[r, :, b] = x[r, :, a] * s + x[r, :, b] * c
    return out


def rows_of(table_row, length, page_rows):
    """Cache rows of a request, in order."""
    return np.array([table_row[j // page_rows] * page_rows + j % page_rows for j in range(length)], dtype=np.int64)


def paged_attention(q, k_cache, v_cache, table, lengths, page_rows, picked=None):
    """q [B, heads, 128] over rows of k_cache, v_cache [rows, kv heads, 128]. Requests of negative length are NaN."""
    B, heads, _ = q.shape
    g = heads // k_cache.shape[1]
    out, lse = np.full(q.shape, math.nan), np.full((heads, B), math.nan)
    for b in range(B):
        if lengths[b] < 0:
            continue
        rows = rows_of(table[b], lengths[b], page_rows)
        for h in range(heads):
            mine = rows
            if picked is not None:
                here = [int(x) for x in picked[b, h // g] if x >= 0]
                mine = rows[np.isin(np.arange(lengths[b]) // page_rows, here)]
            out[b, h], lse[h, b] = attention_row(q[b, h], k_cache[mine, h // g], v_cache[mine, h // g])
    return out, lse


def least_power(top, most):
    """The smallest power of two s >= 2^-126 with top / s <= most; 1 for 0."""
    if top == 0:
        return 1.0
    s = 2.0 ** -126
    while top / s > most:
        s *= 2
    return s


def page_bounds(keys):
    """keys [n, 128] of one page and head, finite or not: codes [2, 128] and their scale."""
    lo, hi = np.zeros(128), np.zeros(128)
    for d in range(128):
        fine = keys[np.isfinite(keys[:, d]), d]
        if len(fine):
            lo[d], hi[d] = fine.min(), fine.max()
    s = least_power(max(np.abs(lo).max(), np.abs(hi).max()), 127)
    return np.stack([np.floor(lo / s), np.ceil(hi / s)]).astype(np.int64), s


def page_scores(q, bounds, scales):
    """q [heads of the group, 128], bounds [pages, 2, 128], scales [pages]: score of each page, exactly."""
    best = np.full(len(bounds), -math.inf)
    for row in q:
        row = np.where(np.isfinite(row), row, 0.0)
        s = least_power(np.abs(row).max(), 127)
        c = np.rint(row / s).astype(np.int64)
        for p in range(len(bounds)):
            total = int(np.maximum(c * bounds[p, 0], c * bounds[p, 1]).sum())
            e = int(math.log2(s)) + int(math.log2(scales[p]))
            best[p] = max(best[p], total * 2.0 ** max(-100, min(100, e)))
    return best


def page_select(scores, first, last, most):
    """Pages taken of len(scores): ascending."""
    n = len(scores)
    if n <= most:
        return list(range(n))
    always = set(range(first)) | set(range(n - last, n))
    rest = sorted((p for p in range(n) if p not in always), key=lambda p: (-scores[p], p))
    return sorted(always | set(rest[:most - len(always)]))


class Pages:
    """A state of page tables, as lists: pages[b] of each request, lengths, refs."""

    def __init__(self, pages, lengths, refs, page_rows, width):
        self.pages, self.lengths, self.refs = [list(p) for p in pages], list(lengths), list(refs)
        self.page_rows, self.width = page_rows, width

    def need(self, n):
        return -(-n // self.page_rows)

    def step(self, source, new):
        """New state, rows of the new tokens (request by request), copied pages, and whether pages ran out."""
        before = self
        out = Pages([], [], before.refs, self.page_rows, self.width)
        for b in range(len(before.pages)):
            for p in before.pages[b][:self.need(before.lengths[b])]:
                out.refs[p] -= 1
        for s in source:
            n = before.lengths[s] if s >= 0 else 0
            out.pages.append(before.pages[s][:self.need(n)] if s >= 0 else [])
            out.lengths.append(n)
            for p in out.pages[-1]:
                out.refs[p] += 1
        grow = [a if n + a <= self.width * self.page_rows else 0 for n, a in zip(out.lengths, new)]
        writes = [pages[-1] if a and n % self.page_rows else None for pages, n, a in zip(out.pages, out.lengths, grow)]
        refs = list(out.refs)
        copies = []
        for b, p in enumerate(writes):  # all that write into a page at once, the last of them apart
            others = [x for x, y in enumerate(writes) if y == p]
            copies.append(p is not None and refs[p] > 1 and not (refs[p] == len(others) and b == others[-1]))
        free = [p for p, r in enumerate(refs) if r <= 0]
        taken, short, pairs, rows = 0, False, [], []
        stay = set()  # pages that a request which found no page for its copy goes on holding
        for b, (n, a) in enumerate(zip(list(out.lengths), grow)):
            wants = self.need(n + a) - (self.need(n) - copies[b]) if a else 0
            fits = not wants or (not short and taken + wants <= len(free))
            if copies[b] and not fits:
                stay.add(writes[b])
            if not fits or (a and not copies[b] and writes[b] in stay):
                short = True
                rows += [-1] * new[b]
                continue
            if not a:
                rows += [-1] * new[b]
                continue
            fresh = free[taken:taken + wants]
            taken += wants
            for p in fresh:
                out.refs[p] = 1
            if copies[b]:
                out.refs[writes[b]] -= 1
                pairs.append((writes[b], fresh[0]))
                out.pages[b] = out.pages[b][:-1]
            out.pages[b] = out.pages[b] + fresh
            out.lengths[b] = n + a
            rows += [out.pages[b][j // self.page_rows] * self.page_rows + j % self.page_rows for j in range(n, n + a)]
        return out, rows, pairs, short

    def compact(self):
        """New state and the moves."""
        used = [p for p, r in enumerate(self.refs) if r > 0]
        u = len(used)
        moves = list(zip([p for p in used if p >= u], [p for p in range(u) if self.refs[p] <= 0]))
        to = dict(moves)
        refs = [max(r, 0) for r in self.refs]
        for a, b in moves:
            refs[a], refs[b] = 0, refs[a]
        return Pages([[to.get(p, p) for p in row] for row in self.pages], self.lengths, refs, self.page_rows, self.width), moves
