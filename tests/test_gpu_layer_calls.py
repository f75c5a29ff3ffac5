"""The layer calls (block codes, their products, residual norms and their gradients) where they are called from: tensors at any address with guarded
surroundings, inputs that the kernel ahead is still writing, tensors of more than 2^31 values."""
import ctypes as C
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding as B
from tests.test_gpu_blocks import _check_product, _plain_codes, _same, _values
from tests.test_gpu_early_launch import late_copy  # noqa: F401
from tests.test_gpu_norm_gradient_edges import _check, _inputs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GUARD = 2.5


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()
    torch.cuda.empty_cache()                      # tens of GB


def _room(shape, dtype, offset):
    """(a buffer of guard values, a tensor in it that begins `offset` elements behind a multiple of 256 bytes)"""
    n, lead = math.prod(shape), 128 + offset
    flat = torch.full((lead + n + 128,), GUARD, dtype=dtype, device="cuda")
    return flat, flat[lead:lead + n].view(shape)


def _untouched(flat, t):
    lead = (t.data_ptr() - flat.data_ptr()) // flat.element_size()
    return bool((flat[:lead] == GUARD).all() and (flat[lead + t.numel():] == GUARD).all())


def _moved(t, offset):
    """A copy of the tensor at such an address; the buffer lives as long."""
    if t is None:
        return None
    return _room(t.shape, t.dtype, offset)[1].copy_(t)


def _backward_into(ctx, d, eps, offset):
    """tc_residual_norms_backward by the C call, its outputs in guarded rooms at the given offset."""
    s, y, gate = d["s"], d["y"], d["gate"]
    at = lambda t: None if t is None else t.data_ptr()                            # noqa: E731
    gate_map = gate if gate is not None and gate.dim() == 4 else None
    p = B._NormParams(at(y), at(d["after"]), at(gate) if gate_map is None else None, at(gate_map), at(d["scale"]), at(d["before"]), eps)
    rooms = {"h": _room(s.shape, s.dtype, offset), "y": _room(s.shape, s.dtype, offset), "scale": _room((1,), F32, offset)}
    for k in ("after", "gate", "before"):
        if d[k] is not None:
            rooms[k] = _room(d[k].shape, d[k].dtype, offset)
    o = {k: v[1].data_ptr() for k, v in rooms.items()}
    g = B._NormGrads(o["h"], o["y"], o["gate"] if gate_map is not None else None, o.get("after"), o.get("gate") if gate_map is None else None, o["scale"], o.get("before"))
    n, c, h, w = s.shape
    t = B._Tensor(s.data_ptr(), n, c, h, w, B.TC_F32 if s.dtype == F32 else B.TC_BF16)
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert B.load_library().tc_residual_norms_backward(ctx.ptr, C.addressof(t), C.addressof(p), at(d["dx"]), at(d["ds"]), C.addressof(g), stream) == 0
    for k, (flat, view) in rooms.items():
        assert _untouched(flat, view), k
    return tc.NormGrads(*[rooms[k][1] if k in rooms else None for k in tc.NormGrads._fields])


# Rows that the ring takes (more than two a block), rows in registers, rows that share warps; even and odd maps, with one tile an SM and more, without one.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(2500, 520, 1, 1), (1300, 2048, 1, 1), (700, 1024, 1, 1), (40, 1024, 1, 1), (301, 64, 1, 1), (301, 256, 1, 1), (2500, 521, 1, 1),
                                   (37, 64, 14, 14), (37, 256, 8, 8), (90, 264, 7, 7), (20, 24, 6, 5), (1, 3000, 4, 4)])
@pytest.mark.parametrize("gate", ["channel", "tensor"])
@pytest.mark.parametrize("of_inputs,of_outputs", [(1, 0), (2, 0), (4, 0), (0, 1), (0, 2), (0, 4), (1, 1), (2, 1), (8, 8)])
def test_gradients_at_any_address(ctx, shape, dtype, gate, of_inputs, of_outputs):
    d = {k: _moved(v, of_inputs) for k, v in _inputs(shape, dtype, gate, True, 6).items()}
    _check(d, _backward_into(ctx, d, 1e-5, of_outputs), 1e-5)


# One input of those that the ring takes where it does not begin at 16 bytes, and one vector.
@pytest.mark.parametrize("name", ["s", "y", "dx", "ds", "gate", "after", "before"])
@pytest.mark.parametrize("shape", [(2500, 1024, 1, 1), (37, 64, 14, 14)])
def test_gradients_with_one_tensor_at_an_odd_address(ctx, name, shape):
    for gate in ("tensor", "channel"):
        d = _inputs(shape, BF16, gate, True, 7)
        d[name] = _moved(d[name], 1)
        _check(d, _backward_into(ctx, d, 1e-5, 0), 1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(2500, 520, 1, 1), (1300, 2048, 1, 1), (40, 1024, 1, 1), (301, 64, 1, 1), (37, 64, 14, 14), (37, 256, 8, 8), (20, 24, 6, 5), (1, 3000, 4, 4)])
@pytest.mark.parametrize("of_inputs,of_outputs", [(1, 0), (2, 0), (4, 0), (0, 1), (0, 2), (0, 4), (2, 1)])
def test_norms_at_any_address(ctx, shape, dtype, of_inputs, of_outputs):
    """The sums as at aligned addresses but for the order of a mean's additions."""
    d = _inputs(shape, dtype, "tensor", True, 8)
    args = lambda m: dict(y=m(d["y"]), after=m(d["after"]), gate=m(d["gate"]), scale=d["scale"], before=m(d["before"]), eps=1e-5)       # noqa: E731
    s, x = (t.double() for t in tc.tc_residual_norms(ctx, d["s"], **args(lambda t: t)))
    (room_s, to_s), (room_x, to_x) = (_room(shape, dtype, of_outputs) for _ in range(2))
    tc.tc_residual_norms(ctx, _moved(d["s"], of_inputs), **args(lambda t: _moved(t, of_inputs)), sum_out=to_s, out=to_x)
    assert _untouched(room_s, to_s) and _untouched(room_x, to_x)
    # each side within (c / 8 + 100) roundings of the branch's terms, and of one step of the type
    k, eps = 2 * (shape[1] / 8 + 100) * 2.0 ** -24, torch.finfo(dtype).eps
    y = d["y"].double()
    branch = (d["scale"].double() * d["gate"].double() * d["after"].double()[None, :, None, None] * y / torch.sqrt((y * y).mean(1, keepdim=True) + 1e-5)).abs()
    assert ((to_s.double() - s).abs() <= branch * k + (s.abs() + branch) * eps).all()
    # x: s is rounded after it is taken, so its error is the branch's alone, through itself and through the mean
    s64 = d["s"].double() + branch * torch.sign(d["gate"].double() * d["after"].double()[None, :, None, None] * y)
    r = 1 / torch.sqrt((s64 * s64).mean(1, keepdim=True) + 1e-5)
    err = branch * k + s64.abs() * 2.0 ** -23
    err = d["before"].double().abs()[None, :, None, None] * (err * r + s64.abs() * r ** 3 * (s64.abs() * err).mean(1, keepdim=True)) + x.abs() * k
    assert ((to_x.double() - x).abs() <= err + (x.abs() + err) * eps).all()


# Rows and maps by every way of the store: pairs of CTAs with TMA, by rows of 16 and 8 bytes and value by value; small tiles, in parts by clusters and through the workspace
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,o,h,w", [(5, 1024, 512, 1, 1), (300, 200, 136, 1, 1), (2000, 1000, 1000, 1, 1), (4100, 256, 2056, 1, 1), (40, 9000, 24, 1, 1),
                                       (30, 64, 200, 14, 14), (100, 130, 520, 8, 8), (64, 320, 1100, 7, 7)])
@pytest.mark.parametrize("square", [True, False])
def test_products_into_any_address(ctx, n, k, o, h, w, dtype, square):
    a = tc.tc_quantize_blocks(ctx, _values((n, k, h, w), 1, dtype))
    b = tc.tc_quantize_blocks(ctx, _values((o, k, 1, 1), 2), square=square)
    bias = torch.randn(o, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    for offset in (0, 1, 2, 4, 8):
        flat, out = _room((n, o, h, w), dtype, offset)
        tc.tc_matmul_blocks(ctx, a, b, bias=_moved(bias, offset), relu=True, out=out)
        _check_product(out, a, b, bias, True)
        assert _untouched(flat, out), offset


# ---- inputs that the kernel ahead writes late --------------------------------------------------
TURNS = 6


def _same_bits(got, want):
    for a, b in zip(got, want):
        if isinstance(a, tc.Blocks):
            assert torch.equal(a.codes.view(torch.uint8)[:, :a.cols], b.codes.view(torch.uint8)[:, :a.cols])
            a, b = ((t.scales if t.square else t.scales[:, :t.rows]) for t in (a, b))
        assert torch.equal(a, b)


def _late(ctx, late_copy, make, call):  # noqa: F811
    """`call(x)` on a tensor that is rewritten 40 us after the call's kernels may start, against calls on tensors that have been there long."""
    inputs = [make(i) for i in range(TURNS)]
    want = [call(x) for x in inputs]
    live = torch.zeros_like(inputs[0])
    got = []
    torch.cuda.synchronize()
    for x in inputs:
        late_copy(live, x, 40)
        got.append(call(live))
    assert tc.tc_get_status(ctx) == 0
    for a, b in zip(got, want):
        _same_bits(a, b)


@pytest.mark.parametrize("shape", [(3, 256, 1, 1), (300, 1024, 1, 1), (20, 64, 14, 14), (16, 40, 7, 7)])
def test_codes_wait_for_the_tensor(ctx, late_copy, shape):  # noqa: F811
    for square in (False, True):
        _late(ctx, late_copy, lambda i: _values(shape, i, BF16), lambda x: [*tc.tc_quantize_blocks(ctx, x, rows="both", square=square), tc.tc_quantize_blocks(ctx, x, square=square)])


@pytest.mark.parametrize("p,k,o,square", [(16, 1024, 512, True), (300, 512, 256, False), (2048, 512, 2048, True), (1024, 512, 4096, False), (64, 16384, 48, False)])
def test_products_wait_for_their_operands(ctx, late_copy, p, k, o, square):  # noqa: F811
    """The codes of one operand come late; the scales are those of all turns."""
    b = tc.tc_quantize_blocks(ctx, _values((o, k, 1, 1), 99), square=square)
    scales = tc.tc_quantize_blocks(ctx, _values((p, k, 1, 1), 98)).scales
    _late(ctx, late_copy, lambda i: tc.tc_quantize_blocks(ctx, _values((p, k, 1, 1), i)).codes.view(torch.uint8),
          lambda codes: [tc.tc_matmul_blocks(ctx, tc.Blocks(codes.view(torch.float8_e4m3fn), scales, k), b, dtype=F32)])


@pytest.mark.parametrize("shape", [(8, 64, 1, 1), (16, 1024, 1, 1), (2500, 1024, 1, 1), (1300, 2048, 1, 1), (20, 64, 14, 14), (16, 40, 7, 7), (8, 3000, 4, 4)])
def test_norms_wait_for_the_tensor(ctx, late_copy, shape):  # noqa: F811
    d = _inputs(shape, BF16, "channel", True, 9)
    args = {k: d[k] for k in ("after", "gate", "scale", "before")}
    make = lambda i: _inputs(shape, BF16, "channel", True, 20 + i)["y"]           # noqa: E731

    def norms(y):
        s, (x, codes) = tc.tc_residual_norms(ctx, d["s"], y, **args, blocks="both")
        return s, x, codes
    _late(ctx, late_copy, make, norms)
    _late(ctx, late_copy, make, lambda y: tc.tc_residual_norms_backward(ctx, d["s"], y, d["dx"], d["ds"], **args))
    # a vector that comes late
    vectors = lambda i: 1 + 0.3 * torch.randn(-(-shape[1] // 4) * 4, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")   # noqa: E731
    _late(ctx, late_copy, vectors, lambda v: tc.tc_residual_norms_backward(ctx, d["s"], d["y"], d["dx"], d["ds"], **{**args, "before": v[:shape[1]]}))


# ---- more than 2^31 values ----------------------------------------------------------------------
ROWS = (524291, 4104, 1, 1)              # 2.15e9 values; a row's first value is the 2^31-th in row 523265
MAPS = (43000, 256, 14, 14)              # 2.16e9


def _tail(shape):
    return 400 if shape[2] == 1 else 3


@pytest.mark.parametrize("shape", [ROWS, MAPS])
def test_codes_of_more_than_2_31_values(ctx, shape):
    x = torch.randn(shape, dtype=BF16, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    pixels, channels = tc.tc_quantize_blocks(ctx, x, rows="both")
    alone = tc.tc_quantize_blocks(ctx, x)
    hw = shape[2] * shape[3]
    last = x[-_tail(shape):]
    m = last.permute(0, 2, 3, 1).reshape(-1, shape[1])
    want = _plain_codes(m, False)
    for b in (pixels, alone):
        _same(tc.Blocks(b.codes[-m.shape[0]:], b.scales[:, b.rows - m.shape[0]:b.rows].contiguous(), shape[1]), want, False)
    p = shape[0] * hw
    first = (p - 1) // 128 * 128 - 128                                            # the last two blocks of pixels
    images = x[first // hw:].permute(1, 0, 2, 3).reshape(shape[1], -1)[:, first - first // hw * hw:]
    codes, scales = _plain_codes(images, False)
    assert torch.equal(channels.codes.view(torch.uint8)[:, first:p], codes.view(torch.uint8)) and torch.equal(channels.scales[-2:, :shape[1]], scales)


@pytest.mark.parametrize("n,k,o,h,w,dtype", [(2 ** 20 + 5, 32, 2056, 1, 1, BF16), (5400, 40, 2048, 14, 14, BF16), (2 ** 20 + 5, 2064, 16, 1, 1, F32), (16, 2064, 2 ** 20 + 5, 1, 1, F32),
                                             (11000, 40, 4001, 7, 7, BF16)])
def test_products_of_more_than_2_31_values(ctx, n, k, o, h, w, dtype):
    a, b = tc.tc_quantize_blocks(ctx, _values((n, k, h, w), 1, BF16)), tc.tc_quantize_blocks(ctx, _values((o, k, 1, 1), 2, BF16))
    out = tc.tc_matmul_blocks(ctx, a, b, shape=(n, h, w), dtype=dtype)
    images = min(n, 2 if h > 1 else 300)
    rows, cols = images * h * w, min(o, 3000)
    part = lambda m, count: tc.Blocks(m.codes[-count:], torch.nn.functional.pad(m.scales[:, m.rows - count:m.rows], (0, -count % 128)), k)           # noqa: E731
    _check_product(out[-images:, -cols:], part(a, rows), part(b, cols))
    _check_product(out[:images, :cols], tc.Blocks(a.codes[:rows], a.scales, k), tc.Blocks(b.codes[:cols], b.scales, k))


@pytest.mark.parametrize("shape", [ROWS, MAPS])
def test_norms_of_more_than_2_31_values(ctx, shape):
    g = torch.Generator(device="cuda").manual_seed(3)
    c, tail = shape[1], _tail(shape)
    s, y = (torch.randn(shape, dtype=BF16, generator=g, device="cuda") for _ in range(2))
    v = _inputs((1, c, 1, 1), BF16, "channel", True, 4)
    args = {k: v[k] for k in ("after", "gate", "scale", "before")}
    end = dict(y=y[-tail:].contiguous(), **args)
    got_s, (got_x, codes) = tc.tc_residual_norms(ctx, s, y, **args, blocks="both", eps=1e-5)
    # the same pixels by themselves: to a step of the type, and a code's
    want_s, want_x = (t.double() for t in tc.tc_residual_norms(ctx, s[-tail:].contiguous(), **end, eps=1e-5))
    for got, want in ((got_s, want_s), (got_x, want_x)):
        assert ((got[-tail:].double() - want).abs() <= want.abs() * 2.0 ** -7 + 1e-5).all()
    rows = tail * shape[2] * shape[3]
    values = tc.Blocks(codes.codes[-rows:], torch.nn.functional.pad(codes.scales[:, codes.rows - rows:codes.rows], (0, -rows % 128)), c).dequantize().double()
    want = want_x.permute(0, 2, 3, 1).reshape(-1, c)
    scales = codes.scales[:, codes.rows - rows:codes.rows].double().t().repeat_interleave(128, 1)[:, :c]
    assert ((values - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, scales * 2.0 ** -10) * 1.01 + want.abs() * 2.0 ** -7).all()
    del got_s, got_x, codes
    # gradients that are zero but for the last pixels: theirs, and the vectors' are of those alone
    dx, ds = torch.zeros_like(s), torch.zeros_like(s)
    for t in (dx, ds):
        t[-tail:] = torch.randn((tail,) + shape[1:], dtype=BF16, generator=g, device="cuda")
    got = tc.tc_residual_norms_backward(ctx, s, y, dx, ds, **args, eps=1e-5)
    assert not got.h[:-tail].any() and not got.y[:-tail].any()
    d = dict(s=s[-tail:], y=y[-tail:], dx=dx[-tail:], ds=ds[-tail:], **args)
    _check(d, got._replace(h=got.h[-tail:], y=got.y[-tail:]), 1e-5)
