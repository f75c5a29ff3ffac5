"""Lists of gradients whose rows could not be numbered in 32 bits are refused on the host: the same tensor may be in a list for the norm many times over."""
import ctypes as C

from paper_1905_10830_b200 import binding as B
from tests.test_blocks_refusals import AT, UNSUPPORTED, ctx, lib  # noqa: F401


def test_lists_of_too_many_values(lib, ctx):  # noqa: F811
    def call(counts, dtype):
        g = (B._Gradient * len(counts))(*[B._Gradient(AT, None, n, dtype) for n in counts])
        return lib.tc_gradient_norm(ctx, C.addressof(g), len(counts), 8 * AT, None)

    # 2^31 rows of 8 KB and more
    for counts in ([1 << 42], [(1 << 42) - 1], [1 << 32] * 1024, [1 << 41, 1], [(1 << 41) + 1]):
        assert call(counts, B.TC_F32) == UNSUPPORTED
        assert call(counts, B.TC_BF16) == UNSUPPORTED
