"""Block-scaled 8-bit matrices (tc_quantize_blocks, tc_matmul_blocks) against plain implementations: codes and scales bit for
bit, products against the sum in 64 bits of the values that the codes stand for."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _values(shape, seed, dtype=F32):
    """Values over many powers of two, a few rows of them large, some zeros."""
    g = _gen(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (shape[0],) + (1,) * (len(shape) - 1), generator=g, device="cuda").float())
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.1, torch.zeros((), device="cuda"), x).to(dtype)


def _matrix(x, kind):
    n, c, h, w = x.shape
    return x.permute(0, 2, 3, 1).reshape(-1, c) if kind == "pixels" else x.permute(1, 0, 2, 3).reshape(c, -1)


def _plain_codes(m, square):
    """Row by row, block by block, in fp32."""
    m = m.float()
    rows, cols = m.shape
    codes = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=m.device)
    scales = []
    per = torch.tensor(1.0 / 448.0, dtype=F32, device=m.device)
    for c0 in range(0, cols, 128):
        part = m[:, c0:c0 + 128]
        amax = part.abs().amax(1)
        if square:
            amax = torch.stack([t.max() for t in amax.split(128)])
        scale = torch.where(amax.isfinite(), amax.clamp_min(2.0 ** -100) * per, float("nan"))
        each = scale.repeat_interleave(128)[:rows] if square else scale
        codes[:, c0:c0 + 128] = (part * torch.reciprocal(each)[:, None]).to(torch.float8_e4m3fn)
        scales.append(scale)
    return codes, torch.stack(scales)


def _same(b, want, square):
    codes, scales = want
    got = b.scales if square else b.scales[:, :b.rows]
    assert torch.equal(got.isnan(), scales.isnan()) and torch.equal(got[~got.isnan()], scales[~scales.isnan()])
    got = b.codes[:, :b.cols].float()
    codes = codes.float()
    assert torch.equal(got.isnan(), codes.isnan()) and torch.equal(got[~got.isnan()], codes[~codes.isnan()])


SHAPES = [(1, 1, 1, 1), (1, 4096, 1, 1), (5, 130, 1, 1), (129, 128, 1, 1), (300, 960, 1, 1), (7, 17, 1, 1), (64, 1000, 1, 1),
          (3, 20, 7, 7), (2, 256, 14, 14), (1, 33, 5, 13), (1, 130, 1, 257), (5, 129, 4, 6), (9, 64, 2, 4), (2, 8, 1, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_codes_are_the_plain_ones(ctx, shape, square, dtype):
    x = _values(shape, sum(shape), dtype)
    want = {k: _plain_codes(_matrix(x, k), square) for k in ("pixels", "channels")}
    both = tc.tc_quantize_blocks(ctx, x, rows="both", square=square)
    for kind, b in zip(("pixels", "channels"), both):
        _same(b, want[kind], square)
        _same(tc.tc_quantize_blocks(ctx, x, rows=kind, square=square), want[kind], square)
    if square:                           # one tile, one scale: the two layouts hold the same values
        assert torch.equal(both[0].codes[:, :both[0].cols].float(), both[1].codes[:, :both[1].cols].float().t())


@pytest.mark.parametrize("shape", [(40, 300, 1, 1), (3, 136, 7, 7), (3, 136, 4, 4), (1, 16, 8, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_codes_of_views_at_any_address_and_of_bad_values(ctx, shape, dtype):
    n = math.prod(shape)
    for offset in (1, 2, 4):
        flat = torch.empty(n + offset, dtype=dtype, device="cuda")
        x = flat[offset:].view(shape)
        x.copy_(_values(shape, 5, dtype))
        for kind in ("pixels", "channels"):
            _same(tc.tc_quantize_blocks(ctx, x, rows=kind), _plain_codes(_matrix(x, kind), False), False)
    x = _values(shape, 6, dtype).contiguous()
    x.view(-1)[[0, n // 3, n // 2, n - 1]] = torch.tensor([float("nan"), float("inf"), float("-inf"), 1e-42], device="cuda").to(dtype)
    x.view(shape)[0, 1] = 0
    for square in (False, True):
        for kind, b in zip(("pixels", "channels"), tc.tc_quantize_blocks(ctx, x, rows="both", square=square)):
            _same(b, _plain_codes(_matrix(x, kind), square), square)


def test_codes_leave_the_rest_of_their_buffers(ctx):
    x = _values((37, 200, 1, 1), 1, BF16)
    b = tc.Blocks.empty(37, 200, device="cuda")
    b.codes.view(torch.uint8).fill_(0x55)
    b.scales.fill_(-7.0)
    assert tc.tc_quantize_blocks(ctx, x, out=b) is b
    assert (b.scales[:, 37:] == -7).all()
    _same(b, _plain_codes(_matrix(x, "pixels"), False), False)


def _operand(rows, cols, seed, square):
    return tc.tc_quantize_blocks(_operand.ctx, _values((rows, cols, 1, 1), seed), square=square)


def _exact(b):
    """The values in 64 bits."""
    s = (b.scales.repeat_interleave(128, 1) if b.square else b.scales)[:, :b.rows].double()
    return b.codes[:, :b.cols].double() * s.t().repeat_interleave(128, 1)[:, :b.cols]


def _check_product(out, a, b, bias=None, relu=False, shape=None):
    va, vb = _exact(a), _exact(b)
    want = va @ vb.t()
    # Products of codes are exact in fp32.  The tensor cores add 32 of them to a block's sum at a time, four times, with at least 22 bits
    # behind the largest term's leading one; the two scales cost two roundings of 2^-24, the sum over the blocks one for each, all
    # relative to the sum of the magnitudes; then the bias and the rounding to the output's type, half a step.
    size = va.abs() @ vb.abs().t()
    blocks = -(-a.cols // 128)
    tol = size * (8 * 2.0 ** -22 + (blocks + 3) * 2.0 ** -24)
    if bias is not None:
        want = want + bias.double()
        tol = tol + want.abs() * 2.0 ** -24
    if relu:
        want = want.clamp_min(0)
    tol = tol + (want.abs() + tol) * torch.finfo(out.dtype).eps / 2 + 1e-38
    got = out.permute(0, 2, 3, 1).reshape(a.rows, b.rows).double()
    bad = (got - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), ((got - want).abs() / tol).max().item())


PRODUCTS = [(1, 1, 1), (1, 128, 16), (3, 200, 5), (17, 129, 127), (128, 128, 256), (130, 384, 257), (64, 4096, 300), (257, 1000, 640),
            (1, 4096, 4096), (2, 960, 1000), (33, 512, 2048), (100, 320, 96), (1000, 64, 64), (3000, 130, 130), (16, 16, 20000),
            (20000, 48, 40), (500, 2000, 500),
            (2100, 300, 1300), (1500, 1000, 2000), (4096, 130, 4096)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("squares", [(False, True), (False, False), (True, False), (True, True)])
@pytest.mark.parametrize("p,k,o", PRODUCTS)
def test_product(ctx, p, k, o, squares, dtype):
    _operand.ctx = ctx
    a, b = _operand(p, k, 1, squares[0]), _operand(o, k, 2, squares[1])
    for bias, relu in ((None, False), (torch.randn(o, generator=_gen(3), device="cuda") * 5, True)):
        _check_product(tc.tc_matmul_blocks(ctx, a, b, dtype=dtype, bias=bias, relu=relu), a, b, bias, relu)


@pytest.mark.parametrize("n,h,w,k,o", [(37, 7, 7, 320, 96), (3, 14, 14, 256, 257), (1, 5, 7, 64, 300), (700, 2, 3, 48, 16), (1, 1, 333, 96, 128), (2, 56, 56, 24, 144),
                                       (40, 7, 7, 200, 1100), (30, 14, 14, 130, 200), (9, 16, 16, 64, 333), (70, 19, 19, 80, 48), (11, 2, 6, 300, 500)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_product_into_maps(ctx, n, h, w, k, o, dtype):
    x = _values((n, k, h, w), 7, dtype)
    a = tc.tc_quantize_blocks(ctx, x)
    b = tc.tc_quantize_blocks(ctx, _values((o, k, 1, 1), 8), square=True)
    bias = torch.randn(o, generator=_gen(3), device="cuda")
    room = torch.full((n * o * h * w + 64,), 3.5, dtype=dtype, device="cuda")
    out = room[32:-32].view(n, o, h, w)
    assert tc.tc_matmul_blocks(ctx, a, b, bias=bias, relu=True, out=out) is out
    _check_product(out, a, b, bias, True)
    assert (room[:32] == 3.5).all() and (room[-32:] == 3.5).all()
    one = tc.tc_matmul_blocks(ctx, a, b, shape=(n, h, w), dtype=dtype, bias=bias, relu=True)
    assert torch.equal(one, out)


@pytest.mark.parametrize("o,c,n,hw", [(40, 56, 3000, 1), (130, 257, 40, 49), (256, 128, 20000, 1), (16, 16, 70000, 1), (300, 520, 1, 1),
                                       (2048, 1500, 700, 1)])
def test_gradient_of_weights(ctx, o, c, n, hw):
    """Long sums with a scale for each row on both sides, taken in parts where the output is small."""
    side = math.isqrt(hw)
    dy, x = _values((n, o, side, side), 11, BF16), _values((n, c, side, side), 12, BF16)
    a, b = tc.tc_quantize_blocks(ctx, dy, rows="channels"), tc.tc_quantize_blocks(ctx, x, rows="channels")
    out = tc.tc_matmul_blocks(ctx, a, b, dtype=F32)
    _check_product(out, a, b)
    again = tc.tc_matmul_blocks(ctx, a, b, dtype=F32)
    assert torch.equal(out, again)
    tc.tc_force_exact_path(ctx, 4)          # no memory for the parts: in one
    try:
        _check_product(tc.tc_matmul_blocks(ctx, a, b, dtype=F32), a, b)
    finally:
        tc.tc_force_exact_path(ctx, 0)


def test_bad_values_stay_in_their_rows(ctx):
    x = _values((200, 300, 1, 1), 21)
    x[5, 7] = float("inf")
    x[140, 299] = float("nan")
    w = _values((70, 300, 1, 1), 22)
    w[3, 0] = float("nan")
    a = tc.tc_quantize_blocks(ctx, x)
    b = tc.tc_quantize_blocks(ctx, w)
    for relu in (False, True):
        bad = tc.tc_matmul_blocks(ctx, a, b, dtype=F32, relu=relu)[:, :, 0, 0].isnan()
        want = torch.zeros_like(bad)
        want[5], want[140], want[:, 3] = True, True, True
        assert torch.equal(bad, want)


def test_padding_is_never_used(ctx):
    """NaN in the padding of codes and scales reaches nothing."""
    for p, k, o, square in ((5, 200, 20, True), (300, 100, 130, False), (17, 130, 16, False)):
        a = tc.tc_quantize_blocks(ctx, _values((p, k, 1, 1), 31))
        b = tc.tc_quantize_blocks(ctx, _values((o, k, 1, 1), 32), square=square)
        for m in (a, b):
            m.codes.view(torch.uint8)[:, m.cols:] = 0x7f
            if not m.square:
                m.scales[:, m.rows:] = float("nan")
        _check_product(tc.tc_matmul_blocks(ctx, a, b, dtype=F32), a, b)


def test_empty(ctx):
    a, b = tc.Blocks.empty(0, 64, device="cuda"), tc.tc_quantize_blocks(ctx, _values((16, 64, 1, 1), 1), square=True)
    assert tc.tc_matmul_blocks(ctx, a, b).shape == (0, 16, 1, 1)
    pixels, channels = tc.tc_quantize_blocks(ctx, torch.empty((0, 64, 1, 1), device="cuda"), rows="both")
    assert (pixels.rows, pixels.cols, channels.rows, channels.cols) == (0, 64, 64, 0)
    dw = tc.tc_matmul_blocks(ctx, channels, tc.Blocks.empty(24, 0, device="cuda"), dtype=F32)   # the gradient of no tokens
    assert dw.shape == (64, 24, 1, 1) and not dw.any()
    bias = torch.randn(24, generator=_gen(1), device="cuda")
    got = tc.tc_matmul_blocks(ctx, channels, tc.Blocks.empty(24, 0, device="cuda"), dtype=F32, bias=bias, relu=True)[:, :, 0, 0]
    assert torch.equal(got, bias.clamp_min(0).expand(64, 24))


def test_captured_and_on_another_stream(ctx):
    """Replays read the buffers' present values; a call between them does not disturb them."""
    x, w = _values((24, 1024, 1, 1), 41, BF16), _values((512, 1024, 1, 1), 42)
    b = tc.tc_quantize_blocks(ctx, w, square=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a = tc.tc_quantize_blocks(ctx, x)
        out = tc.tc_matmul_blocks(ctx, a, b, dtype=F32)
    stream.synchronize()
    _check_product(out, a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tc.tc_quantize_blocks(ctx, x, out=a)
        tc.tc_matmul_blocks(ctx, a, b, out=out)
    for seed in (43, 44):
        x.copy_(_values((24, 1024, 1, 1), seed, BF16))
        other = tc.tc_matmul_blocks(ctx, tc.tc_quantize_blocks(ctx, _values((8, 4096, 1, 1), seed)), tc.tc_quantize_blocks(ctx, _values((300, 4096, 1, 1), 1), square=True))
        graph.replay()
        torch.cuda.synchronize()
        fresh = tc.tc_quantize_blocks(ctx, x)
        assert torch.equal(fresh.codes.view(torch.uint8), a.codes.view(torch.uint8))
        _check_product(out, a, b)
        assert other.isfinite().all()


def test_refusals(ctx):
    a = tc.tc_quantize_blocks(ctx, _values((8, 64, 1, 1), 1))
    b = tc.tc_quantize_blocks(ctx, _values((16, 64, 1, 1), 2), square=True)
    with pytest.raises(tc.TcError):
        tc.tc_matmul_blocks(ctx, a, tc.tc_quantize_blocks(ctx, _values((16, 48, 1, 1), 2)))            # other lengths
    with pytest.raises(tc.TcError):
        tc.tc_matmul_blocks(ctx, a, b, shape=(3, 3, 1))                                                # not a's pixels
    with pytest.raises(ValueError):
        tc.tc_matmul_blocks(ctx, a, b, bias=torch.zeros(15, device="cuda"))
    with pytest.raises(ValueError):
        tc.tc_matmul_blocks(ctx, a, b, dtype=torch.float16)
    with pytest.raises(ValueError):
        tc.tc_matmul_blocks(ctx, tc.Blocks(a.codes, a.scales, 65), b)
    with pytest.raises(ValueError):
        tc.tc_matmul_blocks(ctx, tc.Blocks(a.codes[:, :32], a.scales, 32), b)                          # not contiguous
    with pytest.raises(ValueError):
        tc.tc_quantize_blocks(ctx, _values((8, 64, 1, 1), 1)[:, ::2])
    with pytest.raises(ValueError):
        tc.tc_quantize_blocks(ctx, _values((8, 64, 1, 1), 1), rows="columns")
    with pytest.raises(ValueError):
        tc.tc_quantize_blocks(ctx, _values((8, 64, 1, 1), 1), square=True, out=a)
    with pytest.raises(tc.TcError):
        tc.tc_quantize_blocks(ctx, _values((9, 64, 1, 1), 1), out=a)
    with pytest.raises(ValueError):
        tc.tc_quantize_blocks(ctx, torch.zeros(8, 64, 1, 1))                                           # host memory
