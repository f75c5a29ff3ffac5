"""Rings that a warp fills by asynchronous copies: whichever warp's wait ran out, the one that issued the copies does not leave before those in flight have
landed (or its waits for them have run out too): the block's shared memory goes to another one then."""
import os
import re

from paper_1905_10830_b200 import build


def _code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())


def _block(code, start):
    """The braces that open behind `start`, with what they hold."""
    at = code.index("{", start)
    depth = 0
    for i in range(at, len(code)):
        depth += (code[i] == "{") - (code[i] == "}")
        if depth == 0:
            return code[at:i + 1]
    raise AssertionError("unbalanced")


def test_the_ring_of_the_group_norms():
    code = _code("group_norm.cuh")
    body = _block(code, code.index("void fill(unsigned char *ring"))
    loop = body.index("for (; i < pieces; ++i)")
    issue = _block(body, loop)
    assert "bulk_load" in issue and "return" not in body and issue.count("break;") == 1
    rest = body[body.index(issue) + len(issue):]
    assert re.search(r"for \(int last = max\(i - kSlots, 0\); last < i; \+\+last\) arrived\(&full\[last % kSlots\], last / kSlots & 1\);", rest)
    assert "bulk_load" not in rest


def test_the_rings_of_the_integer_products():
    code = _code("row_matmul.cu")
    producers = [m.start() for m in re.finditer(r"long long issued = 0;", code)]
    assert len(producers) == 2
    for at in producers:
        loop = code.index("for (int u = ", at)
        issue = _block(code, loop)
        assert "tma_load_2d" in issue and "++issued;" in issue
        rest = code[code.index(issue, loop) + len(issue):][:600]
        # not only after a wait of its own that ran out
        wait = re.match(r"\s*if \(!alive\) tc_dev_set_status\(a\.status, TC_ERR_TIMEOUT\);\s*for \(long long i = issued > (S::)?kStages \? issued - (S::)?kStages : 0; i < issued; \+\+i\) mbar_wait_soon\(smem_u32\(&s_(full|empty)\[", rest)
        assert wait, rest


def test_the_last_copies_are_those_that_may_be_in_flight():
    """Slots and phases of the waits, for rings of two to five slots: each slot's last copy, none twice."""
    for slots in range(2, 6):
        for issued in range(0, 23):
            waits = [(i % slots, i // slots & 1) for i in range(max(issued - slots, 0), issued)]
            last = {}
            for i in range(issued):
                last[i % slots] = i // slots & 1
            assert dict(waits) == last and len(waits) == len(last)
