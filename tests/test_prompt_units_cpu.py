"""The hand-over of units between the warps of the prompts' kernel, walked through in every order, with the numbers that the kernel has."""
import os
import re

from paper_2403_10444_b200 import build as bv_build


def numbers():
    with open(os.path.join(bv_build.CSRC, "bv_prompt_tiles.cu")) as f:
        source = f.read()
    told = int(re.search(r"constexpr int kTold = (\d+);", source).group(1))
    marks = re.search(r"constexpr int kUnits = ([^;]+);", source).group(1)
    return told, eval(marks, {"kTold": told})


def clashes(told, marks):
    """A state in which the cleaning warps clear the mark of a unit that the weights of an earlier one still have to read, or None.

    A state is the unit that each of three is at: the loading thread (which has told of it), the cleaning warps, the last warps of the weights (which go through
    units they have no tile of, and so wait for nobody else).  Unit u + 1 is told of once all have heard of unit u + 1 - told; one hears of a unit by going on to it."""
    todo, seen = [(0, 0, 0)], set()
    while todo:
        state = todo.pop()
        if state in seen or state[0] > 4 * told + marks:
            continue
        seen.add(state)
        load, clean, weigh = state
        if clean > weigh and clean % marks == weigh % marks:
            return state
        if load + 1 - told <= min(clean, weigh):
            todo.append((load + 1, clean, weigh))
        if clean < load:
            todo.append((load, clean + 1, weigh))
        if weigh < load:
            todo.append((load, clean, weigh + 1))
    return None


def test_a_units_mark_is_read_before_it_is_cleared():
    assert clashes(*numbers()) is None
    # (and the walk finds it where there are as few marks as units told ahead)
    assert clashes(4, 4) is not None and clashes(4, 5) is None
