"""The oracles of the operators over pages against closed forms and one another (no GPU)."""
from __future__ import annotations

import math
import random

import numpy as np
import pytest

from oracle import llm_oracle, pages_oracle as po

RATE = [10000.0 ** (-j / 64) for j in range(64)]


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_turns_by_complex_numbers_and_back(adjacent):
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((3, 2, 128)), np.array([[0, 7, 1000], [5, -3, 9]])
    axis = [0] * 20 + [1] * 44
    y = po.rotary(x, pos, axis, RATE, adjacent)
    z = x[..., 0::2] + 1j * x[..., 1::2] if adjacent else x[..., :64] + 1j * x[..., 64:]
    z = z * np.exp(1j * np.array([[pos[axis[j], r] * RATE[j] for j in range(64)] for r in range(3)]))[:, None]
    got = y[..., 0::2] + 1j * y[..., 1::2] if adjacent else y[..., :64] + 1j * y[..., 64:]
    assert np.allclose(got, z, rtol=0, atol=1e-13)
    assert np.allclose(po.rotary(y, -pos, axis, RATE, adjacent), x, rtol=0, atol=1e-12)


def test_rotary_products_depend_on_the_distance_only():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 128))
    dot = lambda a, b: float((po.rotary(q, np.array([[a]]), [0] * 64, RATE) * po.rotary(k, np.array([[b]]), [0] * 64, RATE)).sum())
    assert abs(dot(5, 2) - dot(105, 102)) < 1e-10


def test_pages_in_any_order_are_the_rows_in_order():
    rng = np.random.default_rng(2)
    cache_k, cache_v, q = rng.standard_normal((96, 1, 128)), rng.standard_normal((96, 1, 128)), rng.standard_normal((1, 2, 128))
    out, lse = po.paged_attention(q, cache_k, cache_v, [[4, 0, 3]], [37], 16)
    rows = np.r_[64:80, 0:16, 48:53]
    want = llm_oracle.attention_row(q[0, 1], cache_k[rows, 0], cache_v[rows, 0])
    assert np.allclose(out[0, 1], want[0]) and math.isclose(lse[1, 0], want[1])
    some, _ = po.paged_attention(q, cache_k, cache_v, [[4, 0, 3]], [37], 16, np.array([[[2, 0, -1]]]))
    want = llm_oracle.attention_row(q[0, 0], cache_k[np.r_[64:80, 48:53], 0], cache_v[np.r_[64:80, 48:53], 0])
    assert np.allclose(some[0, 0], want[0])


def test_bounds_hold_the_keys_and_scores_hold_the_products():
    rng = np.random.default_rng(3)
    pages = rng.standard_normal((5, 16, 128)) * np.exp(rng.standard_normal((5, 1, 1)))
    q = rng.standard_normal((2, 128))
    made = [po.page_bounds(p) for p in pages]
    for p, (codes, s) in zip(pages, made):
        assert (codes[0] * s <= p.min(0)).all() and (codes[1] * s >= p.max(0)).all() and np.abs(codes).max() <= 127
        assert ((p.min(0) - codes[0] * s) < s).all() and ((codes[1] * s - p.max(0)) < s).all()
    scores = po.page_scores(q, np.stack([c for c, _ in made]), [s for _, s in made])
    for p, score in zip(pages, scores):  # but for the rounding of q: half a step times the sum of magnitudes
        slack = 0.5 * max(po.least_power(np.abs(r).max(), 127) for r in q) * np.abs(p).max(0).sum()
        assert score >= (p @ q.T).max() - slack


def test_selection_takes_the_first_the_last_and_the_best():
    assert po.page_select(np.array([0, 5, 9, 5, 1, 0.0]), 1, 1, 4) == [0, 1, 2, 5]
    assert po.page_select(np.zeros(6), 1, 1, 3) == [0, 1, 5]
    assert po.page_select(np.zeros(3), 1, 1, 3) == [0, 1, 2]
    assert po.page_select(np.array([0, 5, 9, 5, 1, 0.0]), 0, 0, 1) == [2]


def random_state(rng, B, n_pages, width, page_rows):
    """Requests with pages of their own, forked from one another, and pages that something else holds."""
    free, pages, lengths, refs = list(range(n_pages)), [], [], [0] * n_pages
    rng.shuffle(free)
    for b in range(B):
        n = rng.choice([0, 1, page_rows, rng.randint(1, width * page_rows)])
        row = [free.pop() for _ in range(min(len(free), -(-n // page_rows)))]
        n = min(n, len(row) * page_rows)
        if b and rng.random() < 0.4:
            a = rng.randrange(b)
            row, n = list(pages[a]), lengths[a]
        for p in row:
            refs[p] += 1
        pages.append(row)
        lengths.append(n)
    for p in rng.sample(range(n_pages), n_pages // 10):
        refs[p] += 1
    return po.Pages(pages, lengths, refs, page_rows, width)


def holders(state, pinned):
    got = list(pinned)
    for b, row in enumerate(state.pages):
        for p in row[:state.need(state.lengths[b])]:
            got[p] += 1
    return got


@pytest.mark.parametrize("seed", range(40))
def test_steps_keep_count_of_holders_and_move_every_row(seed):
    rng = random.Random(seed)
    state = random_state(rng, rng.randint(1, 9), rng.randint(20, 60), 6, 16)
    pinned = [r - h for r, h in zip(state.refs, holders(state, [0] * len(state.refs)))]
    content = {p: [(p, r) for r in range(16)] for p in range(len(state.refs))}  # what each cache row holds
    for _ in range(4):
        source = [rng.randrange(-1, len(state.pages)) for _ in range(rng.randint(1, 9))]
        new = [rng.choice([0, 1, 1, 5, 20]) for _ in source]
        before = [[content[state.pages[s][j // 16]][j % 16] for j in range(state.lengths[s])] if s >= 0 else [] for s in source]
        state, rows, pairs, _ = state.step(source, new)
        assert state.refs == holders(state, pinned) and min(state.refs) >= 0
        for a, b in pairs:
            content[b] = list(content[a])
        written = [r for r in rows if r >= 0]
        assert len(set(written)) == len(written)  # nobody writes where another does
        for r in written:
            content[r // 16][r % 16] = "new"
        at = 0
        for b, (n, a) in enumerate(zip([len(x) for x in before], new)):
            mine = [content[state.pages[b][j // 16]][j % 16] for j in range(state.lengths[b])]
            assert mine[:n] == before[b] and all(x == "new" for x in mine[n:])
            assert state.lengths[b] in (n, n + a)
            at += a
    used = sum(r > 0 for r in state.refs)
    small, moves = state.compact()
    assert all(r > 0 for r in small.refs[:used]) and not any(small.refs[used:])
    assert len({b for _, b in moves}) == len(moves) and all(a >= used > b for a, b in moves)
