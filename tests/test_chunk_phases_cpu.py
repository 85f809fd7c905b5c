"""The barriers of the chunk attention's scores, in every order of what runs beside one another.

A tile of the bf16 form as its warps run it: an item of n steps has n + 2 entries; entry e waits for P of step e - 2, issues P V of
that step and S of step e, and completes a phase of barrier x % N (x: entries of the tile so far).  A softmax warp waits for
the phase of each step's entry (and, to rescale, for that of the next one), hands over its P, and at the item's end waits for the
last two.  A wait asks for a parity: it may only see its own phase, and that one must not be two phases behind."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_18647_gb300", "csrc")


def programs(items):
    issue, softmax = [], []                     # ("P", number) or ("x", number); the same from the softmax's side
    x = p = 0
    for steps in items:
        for e in range(steps + 2):
            if e >= 2:
                issue.append(("P", p + e - 2))
            issue.append(("x", x + e))
        for j in range(steps):
            softmax.append([("x", x + j)] + ([("x", x + j + 1)] if j else []) + [("P", p + j)])
        softmax.append([("x", x + steps), ("x", x + steps + 1)])
        x, p = x + steps + 2, p + steps
    return issue, [a for group in softmax for a in group], p


def faults(items, barriers, warps=2):
    """The states in which a softmax warp's wait sees another phase than its own, or one that is gone."""
    issue, softmax, _ = programs(items)

    def done(at, kind):                         # phases or P's behind place `at` of a program
        return sum(1 for a in at if a[0] == kind)

    completed = [done(issue[:i], "x") for i in range(len(issue) + 1)]
    handed = [done(softmax[:i], "P") for i in range(len(softmax) + 1)]
    start = (0,) + (0,) * warps
    seen, todo, bad = {start}, [start], set()
    while todo:
        state = todo.pop()
        i, at = state[0], state[1:]
        after = []
        if i < len(issue) and (issue[i][0] == "x" or all(handed[a] > issue[i][1] for a in at)):
            after.append((i + 1,) + at)
        for w, a in enumerate(at):
            if a == len(softmax):
                continue
            kind, number = softmax[a]
            if kind == "x":
                count = completed[i]
                phases = (count - number % barriers + barriers - 1) // barriers if count > number % barriers else 0   # of its barrier
                mine = number // barriers
                passes = phases % 2 != mine % 2
                if passes != (phases > mine):
                    bad.add((number, phases))
                if not passes:
                    continue
            after.append((i,) + at[:w] + (a + 1,) + at[w + 1:])
        if not after and (i < len(issue) or any(a < len(softmax) for a in at)):
            bad.add(("stuck",) + state)
        for s in after:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return bad


ITEMS = [[1], [1, 1, 1], [2, 1, 2], [3, 1, 4, 1], [1, 5, 2, 2, 3], [4, 4, 4]]


@pytest.mark.parametrize("items", ITEMS)
def test_no_wait_is_lapped(items):
    source = open(os.path.join(CSRC, "chunk_attention.cu")).read()
    have = re.search(r"constexpr int CH_SBARS = (\d+);", source)
    assert not faults(items, int(have.group(1)) if have else 2)


def test_two_barriers_would_be():
    """(What the model is there to find.)"""
    assert not faults([4], 2) and faults([1, 1], 2) and faults([4, 4], 2)
