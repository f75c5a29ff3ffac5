"""8-bit integers with a scale for each row (tc_quantize_rows, tc_matmul_rows) against plain implementations, bit for bit: codes are those of the
exact quotient, sums are exact."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from tests.test_gpu_blocks import SHAPES, _gen, _matrix, _values

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _plain_codes(m):
    """(codes, scales) of a matrix: the quotient in 64 bits, which no quotient of two fp32 values that is not a border comes near enough to
    round across one (it is 2^-34 away relative to its size at least)."""
    m = m.float()
    amax = m.abs().amax(1)
    bad = ~amax.isfinite()
    scale = torch.where(bad, float("nan"), (amax.clamp_min(2.0 ** -100).double() / 127.0).float())      # rounded once: no quotient lies near a middle
    codes = (m.double() / scale.double()[:, None]).round()
    return torch.where(bad[:, None], 0.0, codes).to(torch.int8), scale


def _same(r, want):
    codes, scales = want
    assert torch.equal(r.scales.isnan(), scales.isnan()) and torch.equal(r.scales[~r.scales.isnan()], scales[~scales.isnan()])
    assert torch.equal(r.codes[:, :r.cols], codes)


def _last(x):
    return x.contiguous(memory_format=torch.channels_last)


LONG = [(3, 8200, 1, 1), (2, 17000, 1, 1), (2, 16, 130, 150), (1, 3, 200, 201), (300, 2050, 1, 1), (200, 513, 1, 1), (20, 1025, 1, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_codes_are_the_plain_ones(ctx, shape, dtype):
    x = _values(shape, sum(shape), dtype)
    for kind in ("pixels", "channels"):
        want = _plain_codes(_matrix(x, kind))
        _same(tc.tc_quantize_rows(ctx, x, rows=kind), want)
        _same(tc.tc_quantize_rows(ctx, _last(x), rows=kind), want)
    for t in (x, _last(x)):
        for kind, r in zip(("pixels", "channels"), tc.tc_quantize_rows(ctx, t, rows="both")):
            _same(r, _plain_codes(_matrix(x, kind)))


@pytest.mark.parametrize("kind", ["pixels", "channels"])
def test_codes_of_quotients_at_the_borders(ctx, kind):
    """Values within a rounding of (k + 1/2) scale on both sides and on it, for scales that are powers of two and others."""
    rows = []
    for amax in (127.0, 254.0, 1.0, 3.3333333, 0.7, 1e-20, 123456.789, 2.0 ** -100, 3e38):
        scale = (torch.tensor(amax, dtype=F32) / 127.0).double()
        border = ((torch.arange(-127, 127, dtype=torch.float64) + 0.5) * scale).to(F32)
        for step in (-2, -1, 0, 1, 2):
            v = (border.view(torch.int32) + step).view(F32)
            rows.append(torch.cat([v.clamp(-amax, amax), torch.tensor([amax, -amax])]))
    m = torch.stack(rows).cuda()
    x = (m if kind == "pixels" else m.t().contiguous())[:, :, None, None].contiguous()
    _same(tc.tc_quantize_rows(ctx, x, rows=kind), _plain_codes(m))


@pytest.mark.parametrize("shape", [(40, 300, 1, 1), (3, 136, 7, 7), (3, 136, 4, 4), (1, 16, 8, 40), (2, 9000, 1, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_codes_of_views_at_any_address_and_of_bad_values(ctx, shape, dtype):
    n = math.prod(shape)
    for offset in (1, 2, 4):
        flat = torch.empty(n + offset, dtype=dtype, device="cuda")
        x = flat[offset:].view(shape)
        x.copy_(_values(shape, 5, dtype))
        for kind, r in zip(("pixels", "channels"), tc.tc_quantize_rows(ctx, x, rows="both")):
            _same(r, _plain_codes(_matrix(x, kind)))
    x = _values(shape, 6, dtype).contiguous()
    x.view(-1)[[0, n // 3, n // 2, n - 1]] = torch.tensor([float("nan"), float("inf"), float("-inf"), 1e-42], device="cuda").to(dtype)
    x[0, 1] = 0
    x[-1, 2] = 1e-39
    for t in (x, _last(x)):
        for kind, r in zip(("pixels", "channels"), tc.tc_quantize_rows(ctx, t, rows="both")):
            _same(r, _plain_codes(_matrix(x, kind)))


def test_codes_leave_the_rest_of_their_buffers(ctx):
    x = _values((37, 205, 1, 1), 1, BF16)
    r = tc.Rows(torch.full((37, 224), 85, dtype=torch.int8, device="cuda"), torch.empty(37, device="cuda"), 205)
    assert tc.tc_quantize_rows(ctx, x, out=r) is r
    assert (r.codes[:, 208:] == 85).all()
    _same(r, _plain_codes(_matrix(x, "pixels")))


# ---- products ------------------------------------------------------------------------------
def _operand(rows, cols, seed, ld=None):
    """Codes of all values, -128 too, behind `cols` others that count for nothing."""
    g = _gen(seed)
    ld = -(-cols // 16) * 16 if ld is None else ld
    codes = torch.randint(-128, 128, (rows, ld), generator=g, device="cuda", dtype=torch.int8)
    return tc.Rows(codes, torch.exp2(torch.randint(-8, 3, (rows,), generator=g, device="cuda").float()) * (1 + torch.rand(rows, generator=g, device="cuda")), cols)


def _want(a, b, bias, relu, dtype, shape, pad=1 << 14):
    """The definition, step by step; sums of up to 2^53 are exact in 64 bits."""
    sums = torch.zeros(a.rows, b.rows, dtype=torch.float64, device="cuda")
    for k in range(0, a.cols, pad):
        sums += a.codes[:, k:min(a.cols, k + pad)].double() @ b.codes[:, k:min(a.cols, k + pad)].double().t()
    v = sums.float() * a.scales[:, None] * b.scales if a.cols else sums.float()
    if bias is not None:
        v = v + bias
    if relu:
        v = torch.where(v < 0, 0.0, v)
    n, h, w = shape
    return v.to(dtype).reshape(n, h, w, b.rows).permute(0, 3, 1, 2)


def _check(ctx, a, b, dtype=BF16, bias=None, relu=False, shape=None, channels_last=False):
    out = tc.tc_matmul_rows(ctx, a, b, shape=shape, dtype=dtype, bias=bias, relu=relu, channels_last=channels_last)
    want = _want(a, b, bias, relu, dtype, shape or (a.rows, 1, 1))
    assert out.is_contiguous(memory_format=torch.channels_last if channels_last else torch.contiguous_format)
    assert out.shape == want.shape and torch.equal(out, want), (int((out != want).sum()), out.numel())


# one token to many, few and many channels, sums of one code to some thousand, sizes next to the tiles' and odd ones
PRODUCTS = [(1, 1, 1), (1, 4096, 4096), (1, 130, 17), (2, 129, 300), (7, 4096, 96), (16, 256, 1000), (33, 128, 33), (64, 8192, 512), (100, 64, 100), (127, 383, 129),
            (128, 512, 128), (129, 1000, 257), (256, 256, 256), (300, 200, 136), (1000, 96, 1000), (2000, 1000, 1000), (4096, 128, 4096), (5000, 320, 960), (257, 40, 6000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,o", PRODUCTS)
def test_products_are_exact(ctx, n, k, o, dtype):
    a, b = _operand(n, k, 1), _operand(o, k, 2, ld=-(-k // 16) * 16 + 32)
    bias = torch.randn(o, generator=_gen(3), device="cuda")
    _check(ctx, a, b, dtype)
    _check(ctx, a, b, dtype, bias, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("channels_last", [False, True])
@pytest.mark.parametrize("n,h,w,k,o", [(3, 7, 7, 320, 960), (37, 7, 7, 64, 24), (2, 14, 14, 256, 256), (9, 5, 3, 100, 77), (64, 8, 8, 130, 520), (1, 56, 56, 64, 130), (40, 14, 14, 40, 1100)])
def test_products_of_maps(ctx, n, h, w, k, o, dtype, channels_last):
    a, b = _operand(n * h * w, k, 4), _operand(o, k, 5)
    _check(ctx, a, b, dtype, torch.randn(o, generator=_gen(6), device="cuda"), True, (n, h, w), channels_last)
    _check(ctx, a, b, dtype, None, False, (n, h, w), channels_last)


@pytest.mark.parametrize("n,k,o", [(40, 9000, 24), (3, 131008, 130), (5, 300000, 70), (130, 1000000, 3), (1, 4000001, 1), (200, 262144, 300)])
def test_long_sums(ctx, n, k, o):
    """Parts through clusters and the workspace; sums beyond 32 bits."""
    a, b = _operand(n, k, 7), _operand(o, k, 8)
    _check(ctx, a, b, F32)
    a.codes.fill_(-128)
    b.codes.fill_(-128)
    _check(ctx, a, b, F32)
    b.codes.fill_(127)
    _check(ctx, a, b, BF16)


def test_without_a_workspace(ctx):
    tc.tc_force_exact_path(ctx, 4)
    try:
        for n, k, o in ((4, 130944, 3), (300, 9000, 24), (2, 131072, 2), (5, 300000, 70)):        # (the last two need one)
            _check(ctx, _operand(n, k, 9), _operand(o, k, 10), F32)
        x = _values((40, 64, 1, 1), 1)
        _same(tc.tc_quantize_rows(ctx, x, rows="channels"), _plain_codes(_matrix(x, "channels")))
    finally:
        tc.tc_force_exact_path(ctx, 0)


def test_empty_sums_and_bad_scales(ctx):
    bias = torch.randn(40, generator=_gen(1), device="cuda")
    empty = lambda rows: tc.Rows(torch.empty(rows, 0, dtype=torch.int8, device="cuda"), torch.full((rows,), float("nan"), device="cuda"), 0)   # noqa: E731
    out = tc.tc_matmul_rows(ctx, empty(30), empty(40), bias=bias, relu=True, dtype=F32)
    assert torch.equal(out[:, :, 0, 0], bias.clamp_min(0).expand(30, 40))
    assert tc.tc_matmul_rows(ctx, empty(0), empty(40)).shape == (0, 40, 1, 1)
    a, b = _operand(30, 200, 1), _operand(40, 200, 2)
    a.scales[3], b.scales[7], a.scales[5] = float("nan"), float("nan"), float("inf")
    out = tc.tc_matmul_rows(ctx, a, b, dtype=F32, relu=True)[:, :, 0, 0]
    want = _want(a, b, None, True, F32, (30, 1, 1))[:, :, 0, 0]
    assert torch.equal(out.isnan(), want.isnan()) and out[3].isnan().all() and out[:, 7].isnan().all()
    assert torch.equal(out[~out.isnan()], want[~want.isnan()])


def test_layer_and_gradients_by_codes(ctx):
    """The three products of a training step from the codes of their operands: within the codes' half steps of the products of the values."""
    g = _gen(11)
    x, w, dy = (torch.randn(s, generator=g, device="cuda") for s in ((6, 96, 7, 7), (130, 96, 1, 1), (6, 130, 7, 7)))
    px, cx = tc.tc_quantize_rows(ctx, x, rows="both")
    pw, cw = tc.tc_quantize_rows(ctx, w, rows="both")
    py, cy = tc.tc_quantize_rows(ctx, _last(dy), rows="both")
    for a, b, va, vb, shape in ((px, pw, _matrix(x, "pixels"), w[:, :, 0, 0], (6, 7, 7)), (py, cw, _matrix(dy, "pixels"), w[:, :, 0, 0].t(), (6, 7, 7)),
                                (cy, cx, _matrix(dy, "channels"), _matrix(x, "channels"), (130, 1, 1))):
        out = tc.tc_matmul_rows(ctx, a, b, shape=shape, dtype=F32)
        got = out.permute(0, 2, 3, 1).reshape(a.rows, b.rows).double()
        va, vb = va.double(), vb.double()
        half = lambda r: 0.5 * r.scales.double()[:, None] * (1 + 2.0 ** -20)    # noqa: E731
        tol = half(a) @ vb.abs().sum(1)[None] + va.abs().sum(1)[:, None] @ half(b).t() + a.cols * half(a) @ half(b).t() + got.abs() * 2.0 ** -22
        assert ((got - va @ vb.t()).abs() <= tol).all()


def test_refusals(ctx):
    a, b = _operand(8, 64, 1), _operand(16, 64, 2)
    x = _values((8, 64, 1, 1), 1)
    for bad in (dict(shape=(8, 2, 1)), dict(shape=(8, 1)), dict(dtype=torch.float16), dict(bias=torch.zeros(15, device="cuda")), dict(bias=torch.zeros(16)),
                dict(out=torch.empty(8, 15, 1, 1, device="cuda")), dict(out=torch.empty(8, 16, 1, 1)), dict(out=torch.empty(4, 16, 1, 4, device="cuda")[:, :, :, ::2])):
        with pytest.raises((ValueError, tc.TcError)):
            tc.tc_matmul_rows(ctx, a, b, **bad)
    for bad in (tc.Rows(a.codes, a.scales, 80), tc.Rows(a.codes, a.scales[:7], 64), tc.Rows(a.codes.float(), a.scales, 64), tc.Rows(a.codes[:, :40], a.scales, 40), tc.Rows(a.codes.cpu(), a.scales, 64)):
        with pytest.raises((ValueError, tc.TcError)):
            tc.tc_matmul_rows(ctx, bad, b)
    for bad in (dict(rows="rows"), dict(rows=1), dict(rows="both", out=a), dict(out=tc.Rows.empty(9, 64)), dict(out=tc.tc_quantize_blocks(ctx, x))):
        with pytest.raises((ValueError, TypeError, tc.TcError)):
            tc.tc_quantize_rows(ctx, x, **bad)
    for bad in (x.cpu(), x.half(), x[:, ::2], x[:, :, 0, 0], x.transpose(0, 1)):
        with pytest.raises(ValueError):
            tc.tc_quantize_rows(ctx, bad)
