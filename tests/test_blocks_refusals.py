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
    assert call(blocks(0, 64), b, tensor(0, 16)) == OK


def params(**k):
    v = {"y": None, "after": None, "gate": None, "gate_map": None, "scale": None, "before": None, "eps": 1e-6, **k}
    p = B._NormParams(at(v["y"]), v["after"], v["gate"], at(v["gate_map"]), v["scale"], v["before"], v["eps"])
    p.keep = v
    return p


def test_norms(lib, ctx):
    call = lambda h, p, s, x, b=None, cx=ctx: lib.tc_residual_norms(cx, at(h), at(p), at(s), at(x), at(b), None)   # noqa: E731
    t = lambda i, **k: tensor(**{"n": 8, "c": 64, "at": i * AT, **k})                     # noqa: E731
    whole = dict(y=t(2), after=3 * AT, gate=4 * AT, scale=5 * AT, before=6 * AT)
    assert call(t(1), params(**whole), t(7), t(8), None, None) == INVALID
    assert call(t(1), None, t(7), t(8)) == INVALID
    assert call(None, params(**whole), t(7), t(8)) == INVALID
    for change in (dict(eps=-1.0), dict(eps=float("nan")), dict(y=t(2, n=7)), dict(y=t(2, dtype=B.TC_BF16)), dict(gate_map=t(9)), dict(y=None),
                   dict(before=None), dict(gate=None, gate_map=t(9, c=32))):
        assert call(t(1), params(**{**whole, **change}), t(7), t(8)) == INVALID
    p = params(**whole)
    for s, x in ((None, t(8)), (t(7), None), (t(1), t(8)), (t(2), t(8)), (t(7), t(7)), (t(7), t(3)), (t(7, n=9), t(8)), (t(7), t(8, c=65))):
        assert call(t(1), p, s, x) == INVALID
    for b in (blocks(8, 64, True, 9 * AT), blocks(8, 65, False, 9 * AT), blocks(8, 64, False, 7 * AT)):
        assert call(t(1), p, t(7), None, b) == INVALID
    assert call(t(1), params(before=6 * AT), t(7), t(8)) == INVALID                       # a sum of nothing
    wide = dict(c=16385)
    assert call(t(1, **wide), params(before=6 * AT), None, t(8, **wide)) == UNSUPPORTED
    assert call(t(1, n=0), params(before=6 * AT), None, t(8, n=0)) == OK


def test_norms_backward(lib, ctx):
    t = lambda i, **k: tensor(**{"n": 8, "c": 64, "at": i * AT, **k})                     # noqa: E731

    def grads(dh=None, dy=None, dgate_map=None, dafter=None, dgate=None, dscale=None, dbefore=None):
        g = B._NormGrads(at(dh), at(dy), at(dgate_map), dafter, dgate, dscale, dbefore)
        g.keep = dh, dy, dgate_map
        return g

    call = lambda s, p, dx, ds, g, cx=ctx: lib.tc_residual_norms_backward(cx, at(s), at(p), at(dx), at(ds), at(g), None)   # noqa: E731
    whole = dict(y=t(2), after=3 * AT, gate=4 * AT, scale=5 * AT, before=6 * AT)
    out = dict(dh=t(10), dy=t(11), dafter=12 * AT, dgate=13 * AT, dscale=14 * AT, dbefore=15 * AT)
    p = params(**whole)
    assert call(t(1), p, t(7), t(8), grads(**out), None) == INVALID
    assert call(t(1), p, t(7), t(8), None) == INVALID
    assert call(t(1), p, None, t(8), grads(**out)) == INVALID                             # before, and no gradient of x
    assert call(t(1), params(**{**whole, "before": None}), t(7), t(8), grads(**out)) == INVALID
    for change in (dict(dh=None), dict(dy=None), dict(dh=t(1)), dict(dh=t(7)), dict(dy=t(10)), dict(dh=t(10, n=7)), dict(dgate_map=t(16)), dict(dafter=10 * AT)):
        assert call(t(1), p, t(7), t(8), grads(**{**out, **change})) == INVALID
    for without, extra in ((dict(after=None), "dafter"), (dict(gate=None), "dgate")):
        assert call(t(1), params(**{**whole, **without}), t(7), t(8), grads(**out)) == INVALID, extra
    assert call(t(1), params(**{**whole, "gate": None, "gate_map": t(9)}), t(7), t(8), grads(**{**out, "dgate": None})) == INVALID   # its gradient is required
    alone = params(before=6 * AT)
    for bad in (dict(dh=t(10), dy=t(11)), dict(dh=t(10), dscale=14 * AT)):
        assert call(t(1), alone, t(7), None, grads(**bad)) == INVALID
    wide = dict(c=16385)
    assert call(t(1, **wide), alone, t(7, **wide), None, grads(dh=t(10, **wide))) == UNSUPPORTED
