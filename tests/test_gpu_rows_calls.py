"""The calls on 8-bit integers, group norms and gradients where they are called from: outputs at any address with guarded surroundings, inputs that the kernel ahead is still
writing, other streams, graphs, tensors of more than 2^31 values."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from tests import plain_group_norm as plain
from tests.test_gpu_group_norm import _check_backward, _check_forward, _maps, _vectors
from tests.test_gpu_early_launch import late_copy  # noqa: F401
from tests.test_gpu_layer_calls import TURNS, _room, _untouched
from tests.test_gpu_rows import _operand, _plain_codes, _same, _want

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()
    torch.cuda.empty_cache()                      # tens of GB


# Rows and maps by every way of the store: pairs of CTAs with TMA, by rows of 16 and 8 bytes and value by value; small tiles, in parts by clusters and through the workspace
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,o,h,w", [(5, 1024, 512, 1, 1), (300, 200, 136, 1, 1), (2000, 1000, 1000, 1, 1), (4100, 256, 2056, 1, 1), (4100, 2048, 2056, 1, 1), (40, 9000, 24, 1, 1), (256, 40000, 256, 1, 1),
                                       (30, 64, 200, 14, 14), (100, 130, 520, 8, 8), (64, 320, 1100, 7, 7)])
def test_products_into_any_address(ctx, n, k, o, h, w, dtype):
    a, b = _operand(n * h * w, k, 1), _operand(o, k, 2)
    bias = torch.randn(o, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    want = _want(a, b, bias, True, dtype, (n, h, w))
    for offset in (0, 1, 2, 4, 8):
        flat, out = _room((n, o, h, w), dtype, offset)
        tc.tc_matmul_rows(ctx, a, b, bias=bias, relu=True, out=out)
        assert torch.equal(out, want) and _untouched(flat, out), offset
        flat, last = _room((n, h, w, o), dtype, offset)
        tc.tc_matmul_rows(ctx, a, b, bias=bias, relu=True, out=last.permute(0, 3, 1, 2))
        assert torch.equal(last.permute(0, 3, 1, 2), want) and _untouched(flat, last), offset


def _bits(v):
    if isinstance(v, torch.Tensor):
        return [v.contiguous()]
    if isinstance(v, tc.Rows):
        return [v.codes[:, :v.cols].contiguous(), v.scales]
    return [b for x in v if x is not None for b in _bits(x)]


def _late(late_copy, make, call):  # noqa: F811
    """`call(x)` on a tensor that is rewritten 40 us after the call's kernels may start, against calls on tensors that have been there long."""
    inputs = [make(i) for i in range(TURNS)]
    want = [_bits(call(x)) for x in inputs]
    torch.cuda.synchronize()
    x = torch.empty_like(inputs[0], memory_format=torch.preserve_format)
    for i in range(TURNS):
        late_copy(x, inputs[i], 40)
        got = call(x)
        assert all(torch.equal(p, q) for p, q in zip(_bits(got), want[i])), i


@pytest.mark.parametrize("shape", [(1, 4096, 1, 1), (2000, 2048, 1, 1), (300, 520, 1, 1), (30, 64, 7, 7), (20, 136, 8, 8), (5, 40, 40, 40)])
def test_codes_of_late_inputs(ctx, late_copy, shape):  # noqa: F811
    make = lambda i: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")          # noqa: E731
    for kind in ("pixels", "channels", "both"):
        _late(late_copy, make, lambda x: tc.tc_quantize_rows(ctx, x, rows=kind))


@pytest.mark.parametrize("n,k,o", [(4, 4096, 512), (300, 200, 136), (3000, 256, 2056), (3000, 2048, 2056), (256, 40000, 256)])
def test_products_of_late_inputs(ctx, late_copy, n, k, o):  # noqa: F811
    a, b = _operand(n, k, 3), _operand(o, k, 2)
    of = lambda rows: lambda i: _operand(rows, k, 10 + i).codes                    # noqa: E731
    _late(late_copy, of(n), lambda x: tc.tc_matmul_rows(ctx, tc.Rows(x, a.scales, k), b, dtype=F32))
    _late(late_copy, of(o), lambda x: tc.tc_matmul_rows(ctx, a, tc.Rows(x, b.scales, k), dtype=F32))
    vector = lambda rows: lambda i: torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")   # noqa: E731
    _late(late_copy, vector(n), lambda s: tc.tc_matmul_rows(ctx, tc.Rows(a.codes, s, k), b, dtype=F32))
    _late(late_copy, vector(o), lambda s: tc.tc_matmul_rows(ctx, a, tc.Rows(b.codes, s, k), dtype=F32, bias=s))


@pytest.mark.parametrize("shape,groups", [((1, 256, 14, 14), 32), ((40, 64, 28, 28), 8), ((300, 256, 14, 14), 32), ((4, 30, 9, 9), 3)])
def test_norms_of_late_inputs(ctx, late_copy, shape, groups):  # noqa: F811
    make = lambda i: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").contiguous(memory_format=torch.channels_last)   # noqa: E731
    w = torch.rand(shape[1], device="cuda")
    _late(late_copy, make, lambda x: tc.tc_group_norm(ctx, x, groups, weight=w, bias=w, activation="silu", codes="both"))
    x = make(99)
    _, stats = tc.tc_group_norm(ctx, x, groups, weight=w, bias=w)
    _late(late_copy, make, lambda dy: tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=w, activation="silu"))
    _late(late_copy, lambda i: stats * (1 + i), lambda st: tc.tc_group_norm_backward(ctx, x, x, st, weight=w, bias=w))


# Maps whose runs go through rings: threads that are left over, rows of as many vectors as threads and of one more (no ring), pieces that end inside the last round, codes by teams that share pixels
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,groups", [((30, 144, 50, 50), 12), ((200, 520, 19, 21), 65), ((40, 1024, 30, 31), 32), ((20, 1028, 33, 33), 4), ((9, 2048, 41, 41), 32), ((9, 2056, 41, 41), 8),
                                          ((300, 8, 101, 100), 4), ((1, 24, 700, 700), 3)])
def test_long_maps(ctx, shape, groups, dtype):
    x, dy = _maps(shape, sum(shape), dtype), _maps(shape, 7, dtype, 0.1)
    w, b = _vectors(shape[1], 3)
    got = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, activation="silu")
    (y, codes), stats = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, activation="silu", codes="both")
    assert torch.equal(y, got[0]) and torch.equal(stats, got[1])
    _check_forward(got, x, groups, w, b, 1e-5, "silu")
    _check_forward((codes, stats), x, groups, w, b, 1e-5, "silu")
    g = tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=b, activation="silu")
    _check_backward(g, x, dy, stats, groups, w, b, "silu")
    again = tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=b, activation="silu")
    assert all(torch.equal(p, q) for p, q in zip(g, again))


@pytest.mark.parametrize("n", [1000, 3_000_000])
def test_gradients_of_late_inputs(ctx, late_copy, n):  # noqa: F811
    out = torch.empty(n, device="cuda")
    other = torch.ones(50, device="cuda")
    rest = torch.empty(50, device="cuda")
    make = lambda i: torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")              # noqa: E731
    _late(late_copy, make, lambda x: [tc.tc_clip_gradients(ctx, [other, x], 3.0, out=[rest, out]), out.clone()])


def test_on_a_stream_of_their_own(ctx):
    """Behind work on another stream that the call's own waits for."""
    side = torch.cuda.Stream()
    x, w = torch.randn(4000, 512, 1, 1, device="cuda"), torch.randn(256, 512, 1, 1, device="cuda")
    want = tc.tc_matmul_rows(ctx, tc.tc_quantize_rows(ctx, x), tc.tc_quantize_rows(ctx, w), dtype=F32)
    y = torch.zeros_like(x)
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    for _ in range(5):
        big = big @ big / 64
    y.copy_(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = tc.tc_matmul_rows(ctx, tc.tc_quantize_rows(ctx, y), tc.tc_quantize_rows(ctx, w), dtype=F32)
    side.synchronize()
    assert torch.equal(got, want)


def test_captured_calls_have_workspaces_of_their_own(ctx):
    """Calls with parts in a workspace, captured into two graphs and replayed in turn with eager calls between them."""
    r = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(40, 64, 40, 40, generator=r, device="cuda").contiguous(memory_format=torch.channels_last)
    codes = [_operand(256, 40000, 5), _operand(200, 40000, 6)]
    tokens = torch.randn(3000, 2048, 1, 1, generator=r, device="cuda")
    work = [lambda: [tc.tc_matmul_rows(ctx, codes[0], codes[1], dtype=F32), *tc.tc_group_norm(ctx, x, 8, activation="silu")],
            lambda: [*tc.tc_quantize_rows(ctx, tokens, rows="both"), *tc.tc_group_norm_backward(ctx, x, x, torch.ones(40, 4, 2, device="cuda"))]]
    want = [_bits(f()) for f in work]
    graphs, got, side = [], [], torch.cuda.Stream()
    for f in work:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got.append(f())
        graphs.append(graph)
    for _ in range(3):
        for v in got:
            for b in _bits(v):
                b.zero_()
        for g in graphs:
            g.replay()
            work[0]()
        torch.cuda.synchronize()
        for v, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(_bits(v), w))


def test_more_than_2_31_values(ctx):
    c, hw = 1024, 2048
    n = 2 ** 31 // (c * hw) + 3
    x = torch.zeros(n, 32, 64, c, dtype=BF16, device="cuda").permute(0, 3, 1, 2)
    for i in (0, n // 2, n - 1):
        x[i] = torch.randn(c, 32, 64, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").to(BF16)
    w = torch.rand(c, device="cuda")
    y, stats = tc.tc_group_norm(ctx, x, 32, weight=w, bias=w)
    for i in (0, n - 1):
        one, st = tc.tc_group_norm(ctx, x[i:i + 1].clone(memory_format=torch.channels_last), 32, weight=w, bias=w)
        # cut in other ways: each within the bounds of the statistics, of the type a step
        off, rel = plain.stats_tolerance(x[i:i + 1], 32, 1e-5)
        assert ((st[:, :, 0] - stats[i:i + 1, :, 0]).abs() <= 2 * off).all() and ((st[:, :, 1] / stats[i:i + 1, :, 1] - 1).abs() <= 2.1 * rel).all()
        bound = plain.forward_tolerance(x[i:i + 1], 32, w, w, 1e-5, None).reshape(1, c, 32, 64)
        assert ((one.double() - y[i:i + 1].double()).abs() <= 2 * bound + (one.double().abs() + bound) * 2.0 ** -7).all()
    codes = tc.tc_quantize_rows(ctx, x)
    rows = x[-1].permute(1, 2, 0).reshape(-1, c)
    _same(tc.Rows(codes.codes[-hw:], codes.scales[-hw:], c), _plain_codes(rows))
    del y
    b = _operand(40, c, 1)
    out = tc.tc_matmul_rows(ctx, codes, b, shape=(n, 32, 64))
    assert torch.equal(out[-1:], _want(tc.Rows(codes.codes[-hw:], codes.scales[-hw:], c), b, None, False, BF16, (1, 32, 64)))
    del codes, out
    g = tc.tc_group_norm_backward(ctx, x, x, stats, weight=w, bias=w)
    one = tc.tc_group_norm_backward(ctx, x[-1:].clone(memory_format=torch.channels_last), x[-1:].clone(memory_format=torch.channels_last), stats[-1:].clone(), weight=w, bias=w)
    tol = plain.backward_tolerance(x[-1:], x[-1:], 32, stats[-1:, :, 0], stats[-1:, :, 1], w, w, None)[0].reshape(1, c, 32, 64)
    assert ((g.x[-1:].double() - one.x.double()).abs() <= 2 * tol + (one.x.double().abs() + tol) * 2.0 ** -7).all()
    assert math.isfinite(float(g.weight.sum()))
