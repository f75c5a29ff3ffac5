"""Arguments that the layer calls refuse, found on the host before anything is launched: the C ABI with a context that no
check looks into, so that no device is needed."""
import ctypes as C

import pytest

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding as B

OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_1905_10830_b200 import build
    build.build_library()
    return tc.load_library()


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 16)        # zeros; refused calls never look into it


AT = 1 << 40                                      # addresses that nothing reads


def tensor(n, c, h=1, w=1, dtype=B.TC_F32, at=AT):
    return B._Tensor(at, n, c, h, w, dtype)


def blocks(rows, cols, square=False, at=2 * AT, ld=None):
    return B._Blocks(at, at + (1 << 36), -(-cols // 16) * 16 if ld is None else ld, rows, cols, square)


def at(v):
    return None if v is None else C.addressof(v)



def test_quantize(lib, ctx):
    call = lambda x, p, c, cx=ctx: lib.tc_quantize_blocks(cx, at(x), at(p), at(c), None)              # noqa: E731
    x = tensor(8, 64)
    assert call(x, blocks(8, 64), None, None) == INVALID
    assert call(x, None, None) == INVALID
    assert call(None, blocks(8, 64), None) == INVALID
    for bad in (blocks(9, 64), blocks(8, 65), blocks(64, 8), blocks(8, 64, at=2 * AT + 8), blocks(8, 64, ld=72), blocks(8, 64, ld=48),
                B._Blocks(None, 3 * AT, 64, 8, 64, 0), B._Blocks(3 * AT, None, 64, 8, 64, 0), blocks(8, 64, at=AT + 1024)):
        assert call(x, bad, None) == INVALID
    assert call(x, None, blocks(8, 64)) == INVALID
    assert call(x, blocks(8, 64), blocks(64, 8, True, 3 * AT)) == INVALID                 # one square, one not
    assert call(x, blocks(8, 64), blocks(64, 8, False, 2 * AT)) == INVALID                # the same memory
    assert call(tensor(8, 64, at=AT + 2), blocks(8, 64), None) == INVALID                 # not aligned to an element
    assert call(tensor(8, 64, dtype=B.TC_INT8), blocks(8, 64), None) == INVALID
    assert call(tensor(2**21, 1, 64, 64), blocks(8, 64), None) == UNSUPPORTED
    assert call(tensor(1, 2**22 + 1), blocks(1, 2**22 + 1), None) == UNSUPPORTED
    assert call(tensor(0, 64), blocks(0, 64), blocks(64, 0, False, 3 * AT)) == OK         # nothing to do


def test_matmul(lib, ctx):
    call = lambda a, b, out, cx=ctx, bias=None: lib.tc_matmul_blocks(cx, at(a), at(b), bias, 0, at(out), None)   # noqa: E731
    a, b, out = blocks(8, 64), blocks(16, 64, True, 3 * AT), tensor(8, 16)
    assert call(a, b, out, None) == INVALID
    for args in ((None, b, out), (a, None, out), (a, b, None), (a, blocks(16, 48, True, 3 * AT), out), (a, b, tensor(8, 15)), (a, b, tensor(7, 16)),
                 (a, b, tensor(4, 16, 3, 1)), (a, b, tensor(8, 16, at=2 * AT)), (a, b, tensor(8, 16, at=AT + 1)), (a, blocks(16, 64, True, 3 * AT + 4), out)):
        assert call(*args) == INVALID
    assert call(a, b, out, bias=AT) == INVALID                                            # the bias in the output's memory
    assert call(a, b, out, bias=5 * AT + 2) == INVALID
    assert call(blocks(0, 64), b, tensor(0, 16)) == OK


def params(**k):
    v = {"y": None, "after": None, "gate": None, "gate_map": None, "scale": None, "before": None, "eps": 1e-6, **k}
    return B._NormParams(v["y"], v["after"], v["gate"], v["gate_map"], v["scale"], v["before"], v["eps"])


def test_norms(lib, ctx):
    call = lambda h, p, s, x, b=None, cx=ctx: lib.tc_residual_norms(cx, at(h), at(p), s, x, at(b), None)                # noqa: E731
    h = tensor(8, 64)
    whole = dict(y=2 * AT, after=3 * AT, gate=4 * AT, scale=5 * AT, before=6 * AT)
    s, x = 7 * AT, 8 * AT
    assert call(h, params(**whole), s, x, None, None) == INVALID
    assert call(h, None, s, x) == INVALID
    assert call(None, params(**whole), s, x) == INVALID
    for change in (dict(eps=-1.0), dict(eps=float("nan")), dict(gate_map=9 * AT), dict(y=None), dict(before=None), dict(y=2 * AT + 2), dict(after=3 * AT + 1)):
        assert call(h, params(**{**whole, **change}), s, x) == INVALID
    p = params(**whole)
    for to, norm in ((None, x), (s, None), (AT, x), (2 * AT, x), (s, s), (s, 3 * AT), (AT + 8 * 64 * 4 - 4, x), (s + 2, x), (s, x + 1)):
        assert call(h, p, to, norm) == INVALID
    for b in (blocks(8, 64, True, 9 * AT), blocks(8, 65, False, 9 * AT), blocks(8, 64, False, 7 * AT), blocks(9, 64, False, 9 * AT)):
        assert call(h, p, s, None, b) == INVALID
    assert call(h, params(before=6 * AT), s, x) == INVALID                                # a sum of nothing
    assert call(tensor(8, 16385), params(before=6 * AT), None, x) == UNSUPPORTED
    assert call(tensor(0, 64), params(before=6 * AT), None, x) == OK
    assert call(tensor(8, 64, dtype=B.TC_INT8), p, s, x) == INVALID


def test_norms_backward(lib, ctx):
    def grads(dh=None, dy=None, dgate_map=None, dafter=None, dgate=None, dscale=None, dbefore=None):
        return B._NormGrads(dh, dy, dgate_map, dafter, dgate, dscale, dbefore)

    call = lambda s, p, dx, ds, g, cx=ctx: lib.tc_residual_norms_backward(cx, at(s), at(p), dx, ds, at(g), None)        # noqa: E731
    s, dx, ds = tensor(8, 64), 7 * AT, 8 * AT
    whole = dict(y=2 * AT, after=3 * AT, gate=4 * AT, scale=5 * AT, before=6 * AT)
    out = dict(dh=10 * AT, dy=11 * AT, dafter=12 * AT, dgate=13 * AT, dscale=14 * AT, dbefore=15 * AT)
    p = params(**whole)
    assert call(s, p, dx, ds, grads(**out), None) == INVALID
    assert call(s, p, dx, ds, None) == INVALID
    assert call(s, p, None, ds, grads(**out)) == INVALID                                  # before, and no gradient of x
    assert call(s, params(**{**whole, "before": None}), dx, ds, grads(**out)) == INVALID
    for change in (dict(dh=None), dict(dy=None), dict(dh=AT), dict(dh=dx), dict(dy=10 * AT), dict(dgate_map=16 * AT), dict(dafter=10 * AT), dict(dh=10 * AT + 2),
                   dict(dscale=14 * AT + 1)):
        assert call(s, p, dx, ds, grads(**{**out, **change})) == INVALID
    for without in (dict(after=None), dict(gate=None)):
        assert call(s, params(**{**whole, **without}), dx, ds, grads(**out)) == INVALID
    assert call(s, params(**{**whole, "gate": None, "gate_map": 9 * AT}), dx, ds, grads(**{**out, "dgate": None})) == INVALID   # its gradient is required
    alone = params(before=6 * AT)
    for bad in (dict(dh=10 * AT, dy=11 * AT), dict(dh=10 * AT, dscale=14 * AT)):
        assert call(s, alone, dx, None, grads(**bad)) == INVALID
    assert call(tensor(8, 16385), alone, dx, None, grads(dh=10 * AT)) == UNSUPPORTED
