"""Boxes of shared memory that a warp fills in turn and sends out by asynchronous copies: none is filled while a copy from it may still be pending.  The order of
the steps is read from the kernel's source, and the copies are counted for every number of columns behind the last whole tile and for warps behind the last row."""
import os
import re

import pytest

from paper_1905_10830_b200 import build

OUTSIDE = r"if \(first_row >= a\.rows_a \|\| col0 \+ c >= a\.rows_b\) continue;"
STEPS = {"skip": OUTSIDE, "turn": r"turn = \(turn \+ 1\) % kBoxes;", "wait": r"tma_store_wait_read_but_one\(\)", "fill": r"fill_box<T>\(box,", "store": r"tma_store_2d\(",
         "none": r"else if \(a\.store_tma && lane == 0\)\s*tma_store_none\(\);"}
INSIDE = "first_row < a.rows_a && col0 + c < a.rows_b"


def _steps():
    """The steps of a box by rows in their order; a store is "guarded" where it asks for boxes inside the output, and "none" is a group without a copy for the others."""
    code = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "row_matmul.cu")).read())
    body = next(b for b in re.findall(r"^\{$(.*?)^\}", code, re.M | re.S) if "tma_store_wait_read_but_one" in b)
    body = body[body.index("if (a.by_rows)"):]
    body = body[:body.index("store_lanes<")]
    at = sorted((m.start(), name) for name, pattern in STEPS.items() for m in re.finditer(pattern, body))
    names = [name for _, name in at]
    assert [n for n in names if n not in ("skip", "none")] == ["turn", "wait", "fill", "store"], names
    return names, INSIDE in body


def _overwritten(names, guarded, inside):
    """Whether a box is filled under a pending copy, `inside` saying of each turn whether its box lies in the output."""
    turn, pending = 0, []                             # boxes of the groups of copies, the oldest first
    for here in inside:
        box = turn
        for name in names:
            if name == "skip" and not here:
                break
            if name == "turn":
                turn = (turn + 1) % 2
            elif name == "wait":
                pending = pending[-1:]                # all but the newest have been read
            elif name == "fill" and box in pending:
                return True
            elif name == "store" and (here or not guarded):
                pending.append(box)
            elif name == "none" and not here:
                pending.append(None)
    return False


@pytest.mark.parametrize("columns_of_box", [32, 64])      # of fp32, of bf16
def test_no_box_is_filled_under_a_copy(columns_of_box):
    names, guarded = _steps()
    wide = 128 // columns_of_box                          # boxes of a warp's tile
    for rest in range(1, 129):                            # columns of a warp's last tile
        last = [columns_of_box * i < rest for i in range(wide)]
        for tiles in ([last], [[True] * wide, last, [True] * wide], [last, last, last], [last, [False] * wide, last], [[True] * wide, [False] * wide, [True] * wide]):
            assert not _overwritten(names, guarded, [b for t in tiles for b in t] * 2), (rest, tiles)


def test_the_count_sees_a_turn_without_a_copy():
    assert _overwritten(["turn", "wait", "fill", "store"], True, [True, False, True])
    assert not _overwritten(["turn", "wait", "fill", "store"], False, [True, False, True])
    assert not _overwritten(["turn", "wait", "fill", "store", "none"], True, [True, False, True])
    assert not _overwritten(["skip", "turn", "wait", "fill", "store"], True, [True, False, True])
