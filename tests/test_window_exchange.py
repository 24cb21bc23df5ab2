"""What two warps of window_back_kernel exchange behind one barrier a unit, read from the source: the barrier orders a unit's writes before its
reads, but not these before the writes for the next unit, so there are two copies, by turns.

The model plays the element warps' steps in every order that the barriers allow and looks for a read that finds another unit's number."""
import os
import re

from paper_2509_22323_b200 import build


def wrong_reads(copies, units):
    """Two warps, for each unit i: take it (unit i is written once both have left unit i - 2), write to copy i % copies, arrive, wait for the other,
    read the other's, leave.  Whether any order lets a warp read a number that is not of its unit."""
    start = (((0, 0), (0, 0)), ((None,) * copies,) * 2)              # of each warp (unit, step), and its copies' contents
    seen, todo = {start}, [start]
    while todo:
        at, held = todo.pop()
        for w in range(2):
            (i, step), (j, other) = at[w], at[1 - w]
            if i == units:
                continue
            if step == 0:                                            # unit i - 2 has been left by both
                if j < i - 1:
                    continue
            elif step == 2:                                          # the other has arrived for unit i
                if j < i or (j == i and other < 2):
                    continue
            elif step == 3 and held[1 - w][i % copies] != i:
                return True
            mine = held[w]
            if step == 1:
                mine = mine[:i % copies] + (i,) + mine[i % copies + 1:]
            step = (i, step + 1) if step < 3 else (i + 1, 0)
            following = tuple(step if x == w else at[x] for x in range(2)), tuple(mine if x == w else held[x] for x in range(2))
            if following not in seen:
                seen.add(following)
                todo.append(following)
    return False


def test_one_copy_is_not_enough_and_two_are():
    assert wrong_reads(1, 4)
    assert not wrong_reads(2, 6)


def test_the_parts_of_e_go_by_turns():
    with open(os.path.join(build.CSRC, "k10_window_back.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert re.findall(r"float short_of(\S*)\[WARPS\]\[16\];", text) == ["[2]"]
    uses = re.findall(r"ctl->short_of\[([^\]]*)\]", text)
    assert len(uses) == 3 and set(uses) == {"i & 1"}
