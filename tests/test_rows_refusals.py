"""Arguments that the layer calls on 8-bit integers refuse, found on the host before anything is launched: the C ABI with a context that no
check looks into, so that no device is needed."""
import ctypes as C

import pytest

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding as B
from tests.test_blocks_refusals import AT, INVALID, OK, UNSUPPORTED, at, ctx, lib, tensor  # noqa: F401


def rows(n, cols, at=2 * AT, ld=None):
    return B._Rows(at, at + (1 << 36), -(-cols // 16) * 16 if ld is None else ld, n, cols)


def test_quantize(lib, ctx):  # noqa: F811
    call = lambda x, p, c, cx=ctx: lib.tc_quantize_rows(cx, at(x), at(p), at(c), None)                # noqa: E731
    x = tensor(8, 64)
    assert call(x, rows(8, 64), None, None) == INVALID
    assert call(x, None, None) == INVALID
    assert call(None, rows(8, 64), None) == INVALID
    for bad in (rows(9, 64), rows(8, 65), rows(64, 8), rows(8, 64, at=2 * AT + 8), rows(8, 64, ld=72), rows(8, 64, ld=48),
                B._Rows(None, 3 * AT, 64, 8, 64), B._Rows(3 * AT, None, 64, 8, 64), B._Rows(2 * AT, 3 * AT + 2, 64, 8, 64), rows(8, 64, at=AT + 1024)):
        assert call(x, bad, None) == INVALID
    assert call(x, None, rows(8, 64)) == INVALID
    assert call(x, rows(8, 64), rows(64, 8, 2 * AT)) == INVALID                           # the same memory
    assert call(tensor(8, 64, at=AT + 2), rows(8, 64), None) == INVALID                   # not aligned to an element
    assert call(tensor(8, 64, dtype=B.TC_INT8), rows(8, 64), None) == INVALID
    assert call(tensor(2**21, 1, 64, 64), rows(8, 64), None) == UNSUPPORTED
    assert call(tensor(1, 2**22 + 1), rows(1, 2**22 + 1), None) == UNSUPPORTED
    assert call(tensor(0, 64), rows(0, 64), rows(64, 0, 3 * AT)) == OK                    # nothing to do


def test_matmul(lib, ctx):  # noqa: F811
    call = lambda a, b, out, cx=ctx, bias=None: lib.tc_matmul_rows(cx, at(a), at(b), bias, 0, at(out), None)   # noqa: E731
    a, b, out = rows(8, 64), rows(16, 64, 3 * AT), tensor(8, 16)
    assert call(a, b, out, None) == INVALID
    for args in ((None, b, out), (a, None, out), (a, b, None), (a, rows(16, 48, 3 * AT), out), (a, b, tensor(8, 15)), (a, b, tensor(7, 16)),
                 (a, b, tensor(4, 16, 3, 1)), (a, b, tensor(8, 16, at=2 * AT)), (a, b, tensor(8, 16, at=AT + 1)), (a, rows(16, 64, 3 * AT + 4), out)):
        assert call(*args) == INVALID
    assert call(a, b, out, bias=AT) == INVALID                                            # the bias in the output's memory
    assert call(a, b, out, bias=5 * AT + 2) == INVALID
    assert call(rows(0, 64), b, tensor(0, 16)) == OK


def test_the_library_has_what_the_module_asks_for(lib):  # noqa: F811
    module = B._layer_calls()
    assert all(hasattr(lib, name) for name in module.entry_points) and len(set(module.entry_points)) == len(module.entry_points)
    assert {"Rows", "tc_quantize_rows", "tc_matmul_rows"} <= set(dir(tc))
    assert C.sizeof(B._Rows) == 32
    with pytest.raises(ValueError):
        module.init({}, tc.TcError, tc.Blocks, tc.Rows)


def group_params(groups=4, act=0, weight=None, bias=None, eps=1e-5):
    return B._GroupParams(groups, act, weight, bias, eps)


def test_group_norm(lib, ctx):  # noqa: F811
    call = lambda x, p, y, codes=None, stats=None, cx=ctx: lib.tc_group_norm(cx, at(x), at(p), y, at(codes), stats, None)      # noqa: E731
    x, y, p = tensor(8, 64, 3, 3), 2 * AT, group_params()
    assert call(x, p, y, None, None, None) == INVALID
    for args in ((None, p, y), (x, None, y), (x, p, None), (x, p, AT), (x, p, y + 2), (tensor(8, 64, 3, 3, at=AT + 2), p, y), (x, p, y, rows(72, 65, 3 * AT)), (x, p, y, rows(71, 64, 3 * AT)),
                 (x, p, y, rows(72, 64, 2 * AT)), (x, p, y, None, y), (x, p, y, None, 3 * AT + 4), (x, p, None, rows(72, 64, AT))):
        assert call(*args) == INVALID, args
    for bad in (group_params(0), group_params(-1), group_params(5), group_params(128), group_params(act=3), group_params(act=-1), group_params(eps=-1.0), group_params(eps=float("nan")),
                group_params(weight=3 * AT + 2), group_params(bias=2 * AT), group_params(weight=2 * AT + 64)):
        assert call(x, bad, y) == INVALID
    assert call(tensor(1, 8256), p, y) == UNSUPPORTED
    assert call(tensor(2**21, 4, 64, 64), p, 2**20 * AT) == UNSUPPORTED
    assert call(tensor(0, 64, 3, 3), p, None) == OK


def test_group_norm_backward(lib, ctx):  # noqa: F811
    def call(x, p, stats, dy, dx, dw=None, db=None, cx=ctx):
        return lib.tc_group_norm_backward(cx, at(x), at(p), stats, dy, dx, dw, db, None)

    x, p, stats, dy, dx = tensor(8, 64, 3, 3), group_params(weight=5 * AT, bias=6 * AT), 2 * AT, 3 * AT, 4 * AT
    assert call(x, p, stats, dy, dx, cx=None) == INVALID
    for args in ((None, p, stats, dy, dx), (x, None, stats, dy, dx), (x, p, None, dy, dx), (x, p, stats, None, dx), (x, p, stats, dy, None), (x, p, stats, dy, AT), (x, p, stats, dy, dy),
                 (x, p, stats, dy, stats), (x, p, stats + 4, dy, dx), (x, p, stats, dy + 2, dx), (x, p, stats, dy, dx, dx), (x, p, stats, dy, dx, 5 * AT), (x, p, stats, dy, dx, 7 * AT + 2),
                 (x, p, stats, dy, dx, 7 * AT, 7 * AT), (x, group_params(bias=6 * AT), stats, dy, dx, 7 * AT), (x, group_params(weight=5 * AT), stats, dy, dx, 7 * AT, 8 * AT)):
        assert call(*args) == INVALID, args
    assert call(tensor(1, 8256), group_params(), stats, dy, dx) == UNSUPPORTED
    assert call(tensor(0, 64, 3, 3), group_params(), None, None, None) == OK


def test_gradients(lib, ctx):  # noqa: F811
    def call(items, max_norm=1.0, norm=8 * AT, cx=ctx, n=None):
        g = (B._Gradient * max(1, len(items)))(*items)
        return lib.tc_clip_gradients(cx, C.addressof(g), len(items) if n is None else n, max_norm, norm, None)

    ok = B._Gradient(AT, 2 * AT, 100, B.TC_F32)
    assert call([ok], cx=None) == INVALID
    for bad in (B._Gradient(AT, 2 * AT, -1, B.TC_F32), B._Gradient(AT, 2 * AT, 100, B.TC_INT8), B._Gradient(AT + 2, 2 * AT, 100, B.TC_F32), B._Gradient(AT, 2 * AT + 1, 100, B.TC_BF16),
                B._Gradient(None, 2 * AT, 100, B.TC_F32), B._Gradient(AT, None, 100, B.TC_F32), B._Gradient(AT, AT + 4, 100, B.TC_F32), B._Gradient(AT, AT - 396, 100, B.TC_F32)):
        assert call([bad]) == INVALID
        assert call([B._Gradient(3 * AT, 4 * AT, 8, B.TC_BF16), bad]) == INVALID
    assert call([ok], n=-1) == INVALID and call([ok], norm=None) == INVALID and call([ok], norm=8 * AT + 2) == INVALID
    assert call([ok], max_norm=-1.0) == INVALID and call([ok], max_norm=float("nan")) == INVALID
    assert call([ok], norm=AT + 40) == INVALID and call([ok], norm=2 * AT + 396) == INVALID
    for other in (B._Gradient(3 * AT, 2 * AT + 396, 100, B.TC_F32), B._Gradient(2 * AT, 3 * AT, 100, B.TC_F32), B._Gradient(3 * AT, AT, 100, B.TC_F32)):
        assert call([ok, other]) == INVALID and call([other, ok]) == INVALID
    assert call([B._Gradient(AT, AT, 1 << 43, B.TC_BF16)]) == UNSUPPORTED
    assert lib.tc_clip_gradients(ctx, None, 1, 1.0, 8 * AT, None) == INVALID
    assert lib.tc_gradient_norm(ctx, None, 1, 8 * AT, None) == INVALID
    g = B._Gradient(AT, None, 100, B.TC_F32)
    assert lib.tc_gradient_norm(ctx, C.addressof(g), 1, AT + 8, None) == INVALID           # the norm in what is read
