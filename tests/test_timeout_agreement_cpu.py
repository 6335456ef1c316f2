"""What the two softmax groups of the kernel for many drafted rows do when a wait of their block gives up, in every order of
events. No GPU test makes these waits run out: a group that waits for one that has left would hang the GPU.

The model: a scheduler describes pieces one by one; each group waits for a piece's description (which succeeds if it is there, whatever
the abort flag says, and else fails once the flag is up), works, and meets the other group at a barrier that only both together pass.
The flag may go up at any time, after which the scheduler may still describe a piece that it was about to describe.
"""
from __future__ import annotations

PIECES = 3


def steps(state, agree):
    """States one event away. state: (described, flag, group, group), group: (place, piece, word) with the word it brings to a barrier."""
    described, flag, *groups = state
    if described < PIECES:
        yield (described + 1, flag, *groups)
    if not flag:
        yield (described, True, *groups)
    for i, (place, piece, word) in enumerate(groups):
        moved = []
        if place == "find":
            if piece < described:
                moved.append(("met" if agree else "work", piece, True))
            elif piece == PIECES:  # told that there is no more
                moved.append(("met", piece, False) if agree else ("left", piece, False))
            elif flag:
                moved.append(("met", piece, False) if agree else ("left", piece, False))
        elif place == "work":  # its own waits succeed, or fail once the flag is up
            moved.append(("end", piece, True))
            if flag:
                moved.append(("end", piece, False))
        for m in moved:
            yield (described, flag, *[m if k == i else g for k, g in enumerate(groups)])
    (a, piece_a, word_a), (b, piece_b, word_b) = groups
    if a in ("met", "end") and b in ("met", "end"):  # one barrier for both uses
        assert a == b and piece_a == piece_b, "groups met at different places"
        on = word_a and word_b
        after = (("work", piece_a, True) if a == "met" else ("find", piece_a + 1, True)) if on else ("left", piece_a, False)
        yield (described, flag, after, after)


def stuck(agree):
    start = (0, False, ("find", 0, True), ("find", 0, True))
    seen, todo, ends = {start}, [start], []
    while todo:
        state = todo.pop()
        onward = list(steps(state, agree))
        # a scheduler that stops describing and a flag that is up already leave the groups to themselves
        if not any(s[2:] != state[2:] for s in onward) and state[0] == PIECES and state[1]:
            ends.append(state)
        for s in onward:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return [s for s in ends if {g[0] for g in s[2:]} != {"left"}]


def test_groups_that_agree_on_every_piece_leave_together():
    assert stuck(agree=True) == []


def test_the_model_shows_what_happens_without():
    left = stuck(agree=False)
    assert any({g[0] for g in s[2:]} == {"left", "end"} for s in left)  # one waits at the barrier, one has left
