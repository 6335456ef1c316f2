"""Steps of page tables whose pages run out while requests of unequal lengths share a partial page: nobody's rows are given away.

Every cache row's content is followed through the steps; on the GPU the same states against the oracle's lists.
"""
from __future__ import annotations

import os
import random
import sys

import pytest

from oracle import pages_oracle as po

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_pages_oracle_pins import holders

P = 16


def sharers(rng):
    """Requests in groups that share all pages up to the shortest one's last, with lengths apart inside the last page, and few free pages."""
    pages, lengths, n_pages = [], [], 0
    for _ in range(rng.randint(1, 3)):
        full, count = rng.randint(0, 2), rng.randint(1, 5)
        row = list(range(n_pages, n_pages + full + 1))
        n_pages += full + 1
        for _ in range(count):
            pages.append(list(row))
            lengths.append(full * P + rng.randint(1, P))
    order = list(range(len(pages)))
    rng.shuffle(order)
    pages, lengths = [pages[i] for i in order], [lengths[i] for i in order]
    free = rng.choice([0, 0, 1, 2, 5])
    name = rng.sample(range(n_pages + free), n_pages + free)  # pages in any order
    refs = [0] * (n_pages + free)
    for row in pages:
        row[:] = [name[p] for p in row]
        for p in row:
            refs[p] += 1
    if rng.random() < 0.2:
        refs[pages[0][-1]] += 1  # somebody else's too
    return po.Pages(pages, lengths, refs, P, 5)


def some_step(rng, state):
    n = len(state.pages)
    source = rng.choice([list(range(n)), rng.sample(range(n), n), [rng.randrange(-1, n) for _ in range(rng.randint(1, n + 1))]])
    return source, [rng.choice([0, 1, 1, 1, 3, 5, 17]) for _ in source]


def follow(state, content, source, new):
    """A step of the oracle, with what each cache row holds; every request keeps its rows, and those that grow get rows of their own."""
    before = [[content[state.pages[s][j // P]][j % P] for j in range(state.lengths[s])] if s >= 0 else [] for s in source]
    after, rows, pairs, short = state.step(source, new)
    for a, b in pairs:
        content[b] = list(content[a])
    written = [r for r in rows if r >= 0]
    assert len(set(written)) == len(written)
    for i, r in enumerate(rows):
        if r >= 0:
            content[r // P][r % P] = object()
    for b, (was, a) in enumerate(zip(before, new)):
        mine = [content[after.pages[b][j // P]][j % P] for j in range(after.lengths[b])]
        assert mine[:len(was)] == was, (source, new, b)
        assert after.lengths[b] in (len(was), len(was) + a)
    return after, rows, pairs, short


def fresh(state):
    return {p: [(p, r) for r in range(P)] for p in range(len(state.refs))}


@pytest.mark.parametrize("seed", range(300))
def test_sharers_of_unequal_lengths_keep_their_rows(seed):
    rng = random.Random(seed)
    state = sharers(rng)
    pinned = [r - h for r, h in zip(state.refs, holders(state, [0] * len(state.refs)))]
    content = fresh(state)
    for _ in range(4):
        source, new = some_step(rng, state)
        state, *_ = follow(state, content, source, new)
        assert state.refs == holders(state, pinned) and min(state.refs) >= 0


DIRECTED = [  # pages, lengths, refs, steps of (source, new), lengths after each
    ([[0, 1], [0, 1]], [25, 20], [2, 2], [([0, 1], [3, 3])], [[25, 20]]),
    ([[0, 1], [0, 1]], [30, 20], [2, 2], [([0, 1], [3, 1])], [[30, 20]]),
    ([[0], [0]], [10, 10], [2], [([0, 1], [1, 1]), ([1, 0], [1, 1])], [[10, 10], [10, 10]]),
    ([[0], [0]], [10, 12], [2], [([0, 1], [0, 1])], [[10, 12]]),
    # one free page: the first of three gets it, the second is refused, so the third may not keep the page; then the second goes
    ([[0], [0], [0]], [10, 9, 8], [3, 0], [([0, 1, 2], [1, 1, 1]), ([0, -1, 2], [1, 0, 1])], [[11, 9, 8], [12, 0, 9]]),
    # two free pages: all three grow
    ([[0], [0], [0]], [10, 9, 8], [3, 0, 0], [([0, 1, 2], [1, 1, 1])], [[11, 10, 9]]),
    # a refused writer of another page keeps nobody from growing in place
    ([[0], [1, 2], [1, 2], [0, 3]], [10, 20, 18, 18], [2, 2, 2, 1], [([0, 1, 2, 3], [0, 1, 1, 1])], [[10, 20, 18, 19]]),
]


@pytest.mark.parametrize("case", range(len(DIRECTED)))
def test_a_page_is_kept_only_when_all_others_leave_it(case):
    pages, lengths, refs, steps, after = DIRECTED[case]
    state = po.Pages(pages, lengths, refs, P, 4)
    content = fresh(state)
    for (source, new), want in zip(steps, after):
        state, rows, _, short = follow(state, content, source, new)
        assert state.lengths == want
        assert short == (-1 in rows)


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(DIRECTED)))
def test_a_page_is_kept_only_when_all_others_leave_it_on_the_gpu(case):
    from test_gpu_page_tables import same, step
    pages, lengths, refs, steps, _ = DIRECTED[case]
    state = po.Pages(pages, lengths, refs, P, 4)
    for source, new in steps:
        a, st = step(state, source, new)
        state, rows, pairs, short = state.step(source, new)
        same(a, state, rows, pairs)
        assert st == (3 if short else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(40))
def test_sharers_of_unequal_lengths_on_the_gpu(seed):
    from test_gpu_page_tables import same, step
    rng = random.Random(seed)
    state = sharers(rng)
    for _ in range(4):
        source, new = some_step(rng, state)
        a, st = step(state, source, new)
        state, rows, pairs, short = state.step(source, new)
        same(a, state, rows, pairs)
        refused = any((state.lengths[b] + n > state.width * P and n > 0) for b, n in enumerate(new))
        assert st == (3 if short else 0) or refused


@pytest.mark.gpu
@pytest.mark.parametrize("B", [40, 700, 1024])
def test_many_sharers_of_which_some_are_refused_on_the_gpu(B):
    from test_gpu_page_tables import same, step
    rng = random.Random(B)
    last = [rng.randrange(8) for _ in range(B)]  # each keeps one of eight pages with many others
    pages = [[p] for p in last]
    refs = [last.count(p) for p in range(8)] + [0] * (B // 2)
    state = po.Pages(pages, [rng.randint(1, 15) for _ in range(B)], refs, P, 3)
    source, new = list(range(B)), [1] * B
    a, st = step(state, source, new)
    want, rows, pairs, short = state.step(source, new)
    same(a, want, rows, pairs)
    assert short and st == 3
    b, _ = step(state, None, new, in_place=True, source_given=False)
    same(b, want, rows, pairs, in_place=True)
