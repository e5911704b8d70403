"""The waits of the question kernel's byte rings, as a model on the CPU.

A barrier is waited for by the parity of a phase, and says yes if an odd number of phases lies between that one and the one under way.
That is right only for a waiter that knows the phase before to be complete.  The model runs the warp that asks for the bytes of half
steps and the pairs of warps that widen them in every order that their waits allow, bytes arriving in any order, and fails where a
pair goes on although its bytes are not there, or where nobody can go on."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2607_21599_b200", "csrc", "daf_page_attn.cu")


def _constants():
    text = open(SOURCE).read()
    stages = int(re.search(r"constexpr int kQStages = (\d+);", text).group(1))
    full = re.search(r"constexpr int kQFull = (\d+) \* kQStages;", text)
    assert re.search(r"const int turn = \(warp >> 1\) & 1", text) and re.search(r"for \(int t = turn; t < 2 \* n_t; t \+= 2\)", text), "two pairs in turn"
    return stages, stages * int(full.group(1)) if full else stages


def _run(stages, full, turns, steps, before):
    """Every reachable state of one piece of `steps` half steps behind one of `before`; the first fault, or None.

    A state: half steps asked for, which of them have arrived, where each pair is.  What is waited for are `full` barriers in turn for
    the bytes (`before` and what has arrived say how many phases each has completed) and one of `stages` slots to be free."""
    def phases(barrier, arrived):
        return sum(1 for t in range(before) if t % full == barrier) + sum(1 for t in arrived if t % full == barrier)

    def says_yes(barrier, use, arrived):
        start = sum(1 for t in range(before) if t % full == barrier)
        return (phases(barrier, arrived) & 1) != ((start + use) & 1)

    start = (0, frozenset(), tuple(range(turns)))
    seen, todo = {start}, [start]
    while todo:
        asked, arrived, at = state = todo.pop()
        nexts = []
        consumed = {t for k, pos in enumerate(at) for t in range(k, pos, turns)}
        if asked < steps and (asked < stages or asked - stages in consumed):
            nexts.append((asked + 1, arrived, at))
        nexts += [(asked, arrived | {t}, at) for t in range(asked) if t not in arrived]
        for k, t in enumerate(at):
            if t < steps and says_yes(t % full, t // full, arrived):
                if t not in arrived:
                    return f"half step {t} is taken before its bytes are there (asked for: {asked}, there: {sorted(arrived)}, pairs at {at})"
                nexts.append((asked, arrived, at[:k] + (t + turns,) + at[k + 1:]))
        if not nexts and any(t < steps for t in at):
            return f"nobody can go on: {state}"
        for s in nexts:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


def test_the_model_tells_right_from_wrong():
    assert _run(2, 2, 2, 8, 0) is None and _run(4, 4, 2, 10, 3) is None and _run(3, 3, 1, 9, 1) is None
    assert "is taken before its bytes are there" in _run(3, 3, 2, 10, 0)


@pytest.mark.parametrize("before", range(0, 13, 2))
@pytest.mark.parametrize("steps", [2, 4, 8, 14])
def test_bytes_are_there_when_they_are_widened(steps, before):
    stages, full = _constants()
    assert _run(stages, full, 2, steps, before) is None
