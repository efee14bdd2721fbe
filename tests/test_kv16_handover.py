"""The order in which the 16-bit attention's two slots exchange their maxima and sums, of which no run shows reliably that it
holds (a warp would have to be late by some hundred cycles).

A slot that has units in a run waits for their scores, which are computed once both slots have taken over what the run before
left; in a run of one unit the second slot has none, and nothing holds it back.  All interleavings of the two are gone through,
with the number of places that the source has for what changes hands."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_20186_gb300", "csrc", "attention16.cu")


def _wrong_reads(units, places):
    """What a slot may read that is not the other's of the same run: (slot, run, the run that it belongs to).  A slot's steps in
    a run: 0 its units, 1 its numbers down, 2 arrive, 3 wait for the other's arrival and read, 4 done."""
    runs, wrong, seen = len(units), set(), set()
    todo = [(((0, 0), (0, 0)), ())]
    while todo:
        node = todo.pop()
        if node in seen:
            continue
        seen.add(node)
        at, memory = node
        for slot in (0, 1):
            (run, step), (its_run, its_step) = at[slot], at[1 - slot]
            if run == runs:
                continue
            if step == 0 and units[run] > slot and run > 0 and not (its_run > run - 1 or (its_run == run - 1 and its_step == 4)):
                continue  # the scores come when both have read in the run before
            if step == 3 and not (its_run > run or (its_run == run and its_step >= 3)):
                continue
            held = dict(memory)
            if step == 1:
                held[slot, run % places] = run
            if step == 3 and held.get((1 - slot, run % places)) != run:
                wrong.add((slot, run, held.get((1 - slot, run % places))))
            moved = list(at)
            moved[slot] = (run, step + 1) if step < 4 else (run + 1, 0)
            todo.append((tuple(moved), tuple(sorted(held.items()))))
    return wrong


def _places():
    """Places in tensor memory, by the source: stored to and read from by the count of exchanges, modulo so many."""
    with open(SOURCE) as f:
        text = f.read()
    turn = re.search(r"hand = 2 \* \(splits & (\d)\)", text)
    if turn is None:
        return 1
    store, met, load = (text.index(s) for s in ("tmem_st2(scores + hand", "tc_wait_warp(&met, splits & 1)", "(1 - slot) * 128) + hand, other)"))
    assert turn.start() < store < met < load
    return int(turn.group(1)) + 1


@pytest.mark.parametrize("units", [(2, 1), (1, 1, 1, 1), (3, 1, 2, 1, 1, 5), (2, 2, 2)])
def test_a_slot_reads_what_the_other_put_down_in_the_same_run(units):
    assert not _wrong_reads(units, _places())


def test_one_place_is_not_enough():
    assert (0, 0, 1) in _wrong_reads((2, 1), 1)
