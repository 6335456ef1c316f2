"""The loads of the prompt kernel when a wait of its block gives up, in every order of events: none may be on its way when the last
role leaves, since what then lands belongs to the next block. No GPU test makes these waits run out.

The model: a loader issues N copies, each when a ring slot is free; copies land at any time, in order; a reader waits for
each, or gives up once the flag is up, which may happen at any time. The block ends when both have left.
"""
from __future__ import annotations

N, RING = 4, 2


def steps(state, drains):
    """State: (issued, landed, read, flag, loader, reader); roles are "run", "drain" or "left"."""
    issued, landed, read, flag, loader, reader = state
    if not flag:
        yield (issued, landed, read, True, loader, reader)
    if landed < issued:
        yield (issued, landed + 1, read, flag, loader, reader)
    if loader == "run":
        if issued == N:
            yield (issued, landed, read, flag, "drain" if drains == "always" else "left", reader)
        elif issued - read < RING:
            yield (issued + 1, landed, read, flag, loader, reader)
        elif flag:
            yield (issued, landed, read, flag, "drain" if drains else "left", reader)
    if loader == "drain" and landed == issued:
        yield (issued, landed, read, flag, "left", reader)
    if reader == "run":
        if read == N:
            yield (issued, landed, read, flag, loader, "left")
        elif read < landed:
            yield (issued, landed, read + 1, flag, loader, reader)
        elif flag:
            yield (issued, landed, read, flag, loader, "left")


def ends(drains):
    start = (0, 0, 0, False, "run", "run")
    seen, todo, left, stuck = {start}, [start], [], []
    while todo:
        state = todo.pop()
        onward = list(steps(state, drains))
        if state[4:] == ("left", "left"):
            left.append(state)
        elif not onward:
            stuck.append(state)
        for s in onward:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    assert not stuck and left
    return [s for s in left if s[1] < s[0]]


def test_no_copy_is_on_its_way_when_the_block_ends():
    assert ends("always") == []


def test_the_model_shows_copies_that_only_a_waiting_loader_drains():
    assert any(s[0] == N for s in ends("if it gave up itself"))
