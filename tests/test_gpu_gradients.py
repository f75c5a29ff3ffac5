"""tc_gradient_norm and tc_clip_gradients against sums in 64 bits."""
import ctypes as C
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
# eight squares one after the other in fp32 and the sum of four such, half of it by the root; the norm's own rounding
NORM_REL = (0.5 * 10 + 1.5) * U


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _list(sizes, seed, scale=1.0, offsets=(0,)):
    """Tensors of the sizes, types in turn, at the given offsets (elements) from multiples of 256 bytes, and their rooms."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rooms, views = [], []
    for i, n in enumerate(sizes):
        dtype, offset = (F32, BF16)[i % 2], offsets[i % len(offsets)]
        flat = torch.full((n + offset + 64,), 2.5, dtype=dtype, device="cuda")
        view = flat[offset:offset + n]
        view.copy_(torch.randn(n, generator=g, device="cuda") * scale)
        rooms.append((flat, offset, n))
        views.append(view)
    return rooms, views


def _norm(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


def _untouched(rooms):
    return all(bool((f[:o] == 2.5).all() and (f[o + n:] == 2.5).all()) for f, o, n in rooms)


def _check(got, tensors, before, norm, max_norm):
    """Values after the clipping of `before`."""
    exact = _norm(before)
    assert abs(float(norm) - exact) <= exact * NORM_REL + 1e-45
    if exact <= max_norm * (1 - 2 * NORM_REL):
        assert all(torch.equal(a, b) for a, b in zip(got, before))
        return
    for a, b in zip(got, before):
        want = b.double() * (max_norm / exact)
        tol = want.abs() * (NORM_REL + 3 * U)
        assert ((a.double() - want).abs() <= tol + (want.abs() + tol) * torch.finfo(a.dtype).eps / 2 + 1e-45).all()


# one value to several chunks of 32 KB, sizes next to a chunk's
LISTS = [[1], [7], [0, 3, 0], [16384, 1], [16383, 8193, 8192, 8191, 16385], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10] * 4, [100000, 5, 65536, 1000003], [64] * 200, [300] * 1300, [3_000_017, 11]]


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("offsets", [(0,), (1, 3, 0, 5), (2, 4)])
def test_norm_and_clipping(ctx, sizes, offsets):
    rooms, t = _list(sizes, 1, 0.3, offsets)
    before = [v.clone() for v in t]
    exact = _norm(before)
    assert abs(float(tc.tc_gradient_norm(ctx, t)) - exact) <= exact * NORM_REL
    assert all(torch.equal(a, b) for a, b in zip(t, before))
    for max_norm in (0.37 * exact, 2 * exact, 0.0):
        out_rooms, out = _list(sizes, 2, 1.0, offsets)
        norm = tc.tc_clip_gradients(ctx, t, max_norm, out=out)
        _check(out, t, before, norm, max_norm)
        assert all(torch.equal(a, b) for a, b in zip(t, before)) and _untouched(out_rooms)
        shifted_rooms, shifted = _list(sizes, 2, 1.0, (3,))               # other alignments than the inputs'
        tc.tc_clip_gradients(ctx, t, max_norm, out=shifted)
        assert all(torch.equal(a, b) for a, b in zip(shifted, out)) and _untouched(shifted_rooms)
        again = [v.clone() for v in t]
        rooms2, inplace = _list(sizes, 2, 1.0, offsets)
        for a, b in zip(inplace, again):
            a.copy_(b)
        assert torch.equal(tc.tc_clip_gradients(ctx, inplace, max_norm), norm)
        assert all(torch.equal(a, b) for a, b in zip(inplace, out)) and _untouched(rooms2)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e18, 1e25, 1e36])
def test_values_whose_squares_leave_32_bits(ctx, scale):
    for dtype in (F32, BF16):
        g = torch.Generator(device="cuda").manual_seed(3)
        t = [(torch.randn(n, generator=g, device="cuda") * scale).to(dtype) for n in (40000, 7)]
        t.append(torch.zeros(30000, dtype=dtype, device="cuda"))
        exact = _norm(t)
        assert abs(float(tc.tc_gradient_norm(ctx, t)) - exact) <= exact * NORM_REL + 2.0 ** -149
        t.append(torch.full((5,), 1.0, dtype=dtype, device="cuda"))       # next to ordinary ones
        exact = _norm(t)
        assert abs(float(tc.tc_gradient_norm(ctx, t)) - exact) <= exact * NORM_REL


def test_norms_that_are_not_finite_leave_the_values(ctx):
    for bad in (float("nan"), float("inf"), float("-inf")):
        t = [torch.randn(50000, device="cuda"), torch.randn(77, device="cuda").to(BF16)]
        t[1][5] = bad
        before = [v.clone() for v in t]
        out = [torch.empty_like(v) for v in t]
        norm = tc.tc_clip_gradients(ctx, t, 1.0, out=out)
        assert (norm.isnan() if math.isnan(bad) else norm.isinf()).all()
        tc.tc_clip_gradients(ctx, t, 1.0)
        for a, b, c in zip(t, before, out):
            bits = lambda v: v.view(torch.int32 if v.dtype == F32 else torch.int16)       # noqa: E731
            assert torch.equal(bits(a), bits(b)) and torch.equal(bits(c), bits(b))
    big = [torch.full((100,), 3e38, device="cuda")]                        # the norm is beyond fp32
    assert tc.tc_clip_gradients(ctx, big, 1.0).isinf().all() and (big[0] == 3e38).all()
    t = [torch.ones(4, device="cuda")]
    assert float(tc.tc_clip_gradients(ctx, t, float("inf"))) == 2.0 and (t[0] == 1).all()


def test_orders_of_sides_and_empty_lists(ctx):
    assert float(tc.tc_gradient_norm(ctx, [])) == 0.0 and float(tc.tc_clip_gradients(ctx, (), 1.0)) == 0.0
    w = torch.randn(8, 6, 3, 3, device="cuda").contiguous(memory_format=torch.channels_last)
    m = torch.randn(20, 30, device="cuda").t()
    t = [w, m, torch.zeros(0, 5, device="cuda"), torch.tensor(2.0, device="cuda")]
    before = [v.clone() for v in t]
    norm = tc.tc_clip_gradients(ctx, t, 1.0, norm_out=torch.empty(1, device="cuda"))
    _check(t, t, before, norm, 1.0)
    r = torch.ones(3, device="cuda")
    assert math.isclose(float(tc.tc_gradient_norm(ctx, [r, r])), math.sqrt(6), rel_tol=1e-6)      # read twice, counted twice


def test_refusals(ctx):
    a, b = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    for bad in ([a.cpu()], [a.half()], [a[::2]], [a.expand(3, 100)], [None], 5, [a.double()]):
        with pytest.raises((ValueError, TypeError)):
            tc.tc_clip_gradients(ctx, bad, 1.0)
    for out in ([b, b], [], [b.to(BF16)], [b[:99]], [b.reshape(10, 10)], [a[1:]], b.cpu()):
        with pytest.raises((ValueError, TypeError)):
            tc.tc_clip_gradients(ctx, [a], 1.0, out=out)
    for norm in (-1.0, float("nan")):
        with pytest.raises(tc.TcError):
            tc.tc_clip_gradients(ctx, [a], norm)
    for tensors, out in (([a, a], None), ([a, a[50:]], None), ([a[:50], a[49:99]], None), ([a[:50], b[:50]], [b[:50], a[:50]]), ([a, b], [torch.ones(100, device="cuda")] * 2)):
        with pytest.raises(tc.TcError):
            tc.tc_clip_gradients(ctx, tensors, 1.0, out=out)
    with pytest.raises(tc.TcError):
        tc.tc_clip_gradients(ctx, [a], 1.0, norm_out=a[:1])
    with pytest.raises(ValueError):
        tc.tc_gradient_norm(ctx, [a], norm_out=torch.ones(2, device="cuda"))
    assert (a == 1).all() and (b == 1).all()


def test_a_graph_of_its_own_workspace(ctx):
    """Two captured calls and eager ones between their replays."""
    lists = [[torch.randn(n, device="cuda") for n in sizes] for sizes in ((50000, 300, 7), (200000,))]
    outs, norms, graphs = [[torch.empty_like(t) for t in ts] for ts in lists], [torch.empty(1, device="cuda") for _ in lists], []
    side = torch.cuda.Stream()
    for ts, out, norm in zip(lists, outs, norms):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            tc.tc_clip_gradients(ctx, ts, 3.0, out=out, norm_out=norm)
        graphs.append(graph)
    for turn in range(3):
        for ts in lists:
            for t in ts:
                t.normal_()
        for graph in graphs:
            graph.replay()
            tc.tc_gradient_norm(ctx, lists[0])
        torch.cuda.synchronize()
        for ts, out, norm in zip(lists, outs, norms):
            _check(out, ts, ts, norm, 3.0)


def test_more_than_2_31_values(ctx):
    n = 2 ** 31 + 100_003
    t = torch.zeros(n, dtype=BF16, device="cuda")
    t[-1], t[2 ** 31 + 5], t[0] = 3.0, 4.0, 12.0
    assert float(tc.tc_clip_gradients(ctx, [t], 6.5)) == 13.0
    assert float(t[-1]) == 1.5 and float(t[2 ** 31 + 5]) == 2.0 and float(t[0]) == 6.0
    del t
    torch.cuda.empty_cache()


def test_the_c_call_reads_its_list_before_it_returns(ctx):
    t = torch.full((1000,), 2.0, device="cuda")
    norm = torch.empty(1, device="cuda")
    g = (B._Gradient * 1)(B._Gradient(t.data_ptr(), t.data_ptr(), 1000, B.TC_F32))
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert B.load_library().tc_clip_gradients(ctx.ptr, C.addressof(g), 1, 1.0, norm.data_ptr(), stream) == 0
    g[0] = B._Gradient(None, None, 0, 0)
    torch.cuda.synchronize()
    assert math.isclose(float(norm), 2 * math.sqrt(1000), rel_tol=1e-6) and math.isclose(float(t.norm()), 1.0, rel_tol=1e-5)
