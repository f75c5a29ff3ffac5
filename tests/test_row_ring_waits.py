"""The rings of rows in the residual norms' kernels after a wait that ran out: no copy goes to a slot whose last one may still be in flight, and the
block does not end before those in flight have landed (or their waits have run out too)."""
import os
import re

from paper_1905_10830_b200 import build


def _kernels():
    code = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "residual_norms.cu")).read())
    return [body for body in re.findall(r"^\{$(.*?)^\}", code, re.M | re.S) if "RowReader<" in body]


def test_copies_after_a_wait_that_ran_out():
    kernels = _kernels()
    assert len(kernels) == 2
    for body in kernels:
        brings = re.findall(r"if \(([^;{}]*)\)\s*reader\.bring\(", body)
        assert len(brings) == body.count("reader.bring(") == 1
        assert "reader.alive" in brings[0]
        loop_end = body.rindex("if (++slot == r.stages) slot = 0;")
        assert "reader.finish(r);" in body[loop_end:]
