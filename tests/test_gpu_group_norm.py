"""tc_group_norm and tc_group_norm_backward against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from tests import plain_group_norm as plain

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ACTS = [None, "relu", "silu"]


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _rand(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda")


def _last(x):
    return x.contiguous(memory_format=torch.channels_last)


def _maps(shape, seed, dtype, mean=0.5):
    """Channels of unequal spread and mean, channels_last."""
    r, (n, c, h, w) = _rand(seed), shape
    return (r(n, h, w, c) * torch.exp(0.7 * r(c)) + mean * r(c)).to(dtype).permute(0, 3, 1, 2)


def _vectors(c, seed):
    r = _rand(seed)
    return 1 + 0.3 * r(c), 0.3 * r(c)


def _rounding(dtype, want):
    return want.abs() * torch.finfo(dtype).eps / 2


def _check_forward(got, x, groups, w, b, eps, kind):
    y, stats = got
    one = torch.ones(x.shape[1], device="cuda")
    w, b = one if w is None else w, 0 * one if b is None else b
    mean, rstd = plain.stats(x, groups, eps)
    off, rel = plain.stats_tolerance(x, groups, eps)
    assert stats.shape == (x.shape[0], groups, 2)
    known = rstd.isfinite()                       # (a group of equal values with eps = 0: the definition is 1 / 0, which bounds nothing)
    assert ((stats[:, :, 0].double() - mean).abs() <= off).all() and (((stats[:, :, 1].double() / rstd - 1).abs() <= rel) | ~known).all()
    want, tol = plain.forward(x, groups, w, b, eps, kind)[0], plain.forward_tolerance(x, groups, w, b, eps, kind)
    if isinstance(y, tc.Rows):
        rows = lambda t: t.reshape(x.shape).permute(0, 2, 3, 1).reshape(-1, x.shape[1])      # noqa: E731
        want, tol = rows(want), rows(tol)
        amax, at = want.abs().max(1).values, tol.max(1).values
        assert ((y.scales.double() - amax.clamp_min(2.0 ** -100) / 127).abs() <= at / 127 + y.scales.double() * plain.U * 2).all()
        off = (y.codes[:, :y.cols].double() * y.scales.double()[:, None] - want).abs()
        assert (off <= tol + 0.5 * y.scales.double()[:, None] * (1 + 4 * plain.U)).all()
        return
    assert y.dtype == x.dtype and y.shape == x.shape and y.is_contiguous(memory_format=torch.channels_last)
    off = (plain.grouped(y, groups) - want).abs()
    tol = tol + _rounding(x.dtype, want.abs() + tol) + 1e-38
    assert ((off <= tol) | ~known[:, :, None, None, None]).all(), (int((off > tol).sum()), (off / tol).max().item())


# On a cluster's shared memory (one block a map to eight), in three kernels (maps that do not fit, channels that do not begin at 16 bytes), a
# thread's channels in one group and in several, more channels than threads, groups of one channel and of all.
SHAPES = [((1, 8, 1, 1), 1), ((1, 256, 14, 14), 32), ((3, 320, 7, 7), 32), ((37, 64, 8, 8), 8), ((5, 256, 14, 14), 256), ((2, 96, 20, 20), 1), ((300, 128, 1, 1), 4),
          ((2, 30, 9, 9), 3), ((2, 33, 5, 13), 33), ((7, 17, 3, 3), 1), ((1, 4096, 3, 3), 32), ((1, 8192, 2, 2), 8192), ((2, 2056, 5, 5), 257), ((1, 1000, 40, 40), 10),
          ((1, 64, 160, 160), 32), ((2, 8, 200, 200), 2), ((1, 512, 64, 64), 32), ((9, 48, 28, 28), 4), ((1, 7, 1, 1), 7), ((160, 40, 7, 7), 8), ((4, 12, 1, 300), 4)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_values_and_statistics(ctx, shape, groups, kind, dtype):
    x = _maps(shape, sum(shape), dtype)
    w, b = _vectors(shape[1], 3)
    got = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, eps=1e-5, activation=kind)
    _check_forward(got, x, groups, w, b, 1e-5, kind)
    again = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, eps=1e-5, activation=kind)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    for codes in (True, "both"):
        y, stats = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, eps=1e-5, activation=kind, codes=codes)
        assert torch.equal(stats, got[1])
        if codes == "both":
            assert torch.equal(y[0], got[0])
            y = y[1]
        _check_forward((y, stats), x, groups, w, b, 1e-5, kind)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,groups", SHAPES[1:5] + [((2, 30, 9, 9), 3), ((1, 64, 160, 160), 32)])
def test_without_vectors_and_far_means(ctx, shape, groups, dtype):
    x = _maps(shape, 5, dtype, mean=300.0)
    _check_forward(tc.tc_group_norm(ctx, x, groups), x, groups, None, None, 1e-5, None)
    w, b = _vectors(shape[1], 3)
    _check_forward(tc.tc_group_norm(ctx, x, groups, bias=b, eps=1.0), x, groups, None, b, 1.0, None)
    _check_forward(tc.tc_group_norm(ctx, x, groups, weight=w, eps=0.0, activation="silu"), x, groups, w, None, 0.0, "silu")


def _check_backward(g, x, dy, stats, groups, w, b, kind):
    one = torch.ones(x.shape[1], device="cuda")
    args = (x, dy, groups, stats[:, :, 0], stats[:, :, 1], one if w is None else w, 0 * one if b is None else b, kind)
    want, tol = plain.backward(*args), plain.backward_tolerance(*args)
    assert g.x.dtype == x.dtype and g.x.is_contiguous(memory_format=torch.channels_last)
    off, bound = (plain.grouped(g.x, groups) - want[0]).abs(), tol[0] + _rounding(x.dtype, want[0].abs() + tol[0]) + 1e-38
    assert (off <= bound).all(), (int((off > bound).sum()), (off / bound).max().item())
    for got, given, i in ((g.weight, w, 1), (g.bias, b, 2)):
        assert (got is None) == (given is None)
        if got is not None:
            assert ((got.double() - want[i]).abs() <= tol[i] + want[i].abs() * plain.U).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_gradients(ctx, shape, groups, kind, dtype):
    x, dy = _maps(shape, sum(shape), dtype), _maps(shape, 7, dtype, 0.1)
    w, b = _vectors(shape[1], 3)
    _, stats = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, activation=kind)
    g = tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=b, activation=kind)
    _check_backward(g, x, dy, stats, groups, w, b, kind)
    again = tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=b, activation=kind)
    assert all(torch.equal(p, q) for p, q in zip(g, again))


@pytest.mark.parametrize("given", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("shape,groups", [((3, 320, 7, 7), 32), ((2, 30, 9, 9), 3), ((1, 64, 160, 160), 32)])
def test_gradients_without_vectors(ctx, shape, groups, given):
    x, dy = _maps(shape, 1, F32), _maps(shape, 2, F32)
    w, b = (v if g else None for v, g in zip(_vectors(shape[1], 3), given))
    _, stats = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, activation="silu")
    _check_backward(tc.tc_group_norm_backward(ctx, x, dy, stats, weight=w, bias=b, activation="silu"), x, dy, stats, groups, w, b, "silu")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,groups", [((3, 320, 7, 7), 32), ((1, 64, 160, 160), 32), ((2, 4, 3, 3), 2)])
@pytest.mark.parametrize("offset", [1, 2, 4])
def test_any_address(ctx, shape, groups, dtype, offset):
    """Tensors that begin anywhere, in rooms whose surroundings stay as they were."""
    n, c, h, w = shape

    def room(src=None):
        flat = torch.full((math.prod(shape) + 64,), 2.5, dtype=dtype, device="cuda")
        view = flat[32 + offset:32 + offset + math.prod(shape)].view(n, h, w, c).permute(0, 3, 1, 2)
        return flat, view if src is None else view.copy_(src)

    def untouched(flat):
        return bool((flat[:32 + offset] == 2.5).all() and (flat[32 + offset + math.prod(shape):] == 2.5).all())

    weight, bias = (torch.cat([torch.zeros(offset, device="cuda"), v])[offset:] for v in _vectors(c, 3))
    plain_x, plain_dy = _maps(shape, 1, dtype), _maps(shape, 2, dtype)
    (_, x), (_, dy), (flat, out) = room(plain_x), room(plain_dy), room()
    for source in (x, plain_x):
        y, stats = tc.tc_group_norm(ctx, source, groups, weight=weight, bias=bias, activation="relu", out=out)
        assert y is out and untouched(flat)
        _check_forward((y, stats), x, groups, weight, bias, 1e-5, "relu")
    for p, q in ((x, dy), (plain_x, dy), (x, plain_dy)):
        _check_backward(tc.tc_group_norm_backward(ctx, p, q, stats, weight=weight, bias=bias), x, dy, stats, groups, weight, bias, None)


def test_bad_values_stay_in_their_groups(ctx):
    for shape in ((2, 64, 14, 14), (2, 63, 14, 14), (1, 64, 160, 160)):
        x = _maps(shape, 1, F32).clone()
        groups, c = (8, 64) if shape[1] == 64 else (9, 63)
        x[0, 3, 2, 2], x[-1, c - 1, 1, 1] = float("nan"), float("inf")
        y, stats = tc.tc_group_norm(ctx, x, groups, activation="silu")
        bad = torch.zeros(shape[0], groups, dtype=torch.bool, device="cuda")
        bad[0, 0] = bad[-1, groups - 1] = True
        assert torch.equal(stats.isnan().any(2) | ~stats.isfinite().all(2), bad)
        assert torch.equal(plain.grouped(y, groups).isnan().any(2).any(2).any(2), bad)
        good = torch.where(x.isfinite(), x, torch.zeros((), device="cuda"))
        y0, _ = tc.tc_group_norm(ctx, good, groups, activation="silu")
        assert torch.equal(plain.grouped(y, groups)[~bad], plain.grouped(y0, groups)[~bad])
        (codes, _) = tc.tc_group_norm(ctx, x, groups, codes=True)
        rows = x.permute(0, 2, 3, 1).reshape(-1, c)
        hit = torch.zeros(shape[0], shape[2] * shape[3], dtype=torch.bool, device="cuda")
        hit[0] = hit[-1] = True
        assert torch.equal(codes.scales.isnan(), hit.flatten()) and len(rows) == codes.rows


def test_constant_groups(ctx):
    x = torch.full((2, 16, 5, 5), 3.0, device="cuda").contiguous(memory_format=torch.channels_last)
    w, b = _vectors(16, 1)
    y, stats = tc.tc_group_norm(ctx, x, 4, weight=w, bias=b, eps=1e-4)
    assert torch.equal(y, b[None, :, None, None].expand_as(y)) and torch.equal(stats[:, :, 0], torch.full((2, 4), 3.0, device="cuda"))
    assert torch.allclose(stats[:, :, 1], torch.full((2, 4), 100.0, device="cuda"), rtol=1e-6)


def test_empty(ctx):
    x = torch.empty(0, 16, 5, 5, device="cuda").contiguous(memory_format=torch.channels_last)
    w, b = _vectors(16, 1)
    y, stats = tc.tc_group_norm(ctx, x, 4, weight=w, bias=b)
    assert y.shape == x.shape and stats.shape == (0, 4, 2)
    g = tc.tc_group_norm_backward(ctx, x, torch.empty_like(x), stats, weight=w, bias=b)
    assert g.x.shape == x.shape and not g.weight.any() and not g.bias.any()


def test_refusals(ctx):
    x = _maps((2, 16, 5, 5), 1, F32)
    w, b = _vectors(16, 1)
    y, stats = tc.tc_group_norm(ctx, x, 4)
    for bad in (x.contiguous(), x.half(), x.cpu(), x[:, :, 0], x[:, :8]):
        with pytest.raises(ValueError):
            tc.tc_group_norm(ctx, bad, 4)
    for groups in (0, 3, -4, 32, 1 << 40):
        with pytest.raises(ValueError):
            tc.tc_group_norm(ctx, x, groups)
    for bad in (dict(weight=w[:15]), dict(bias=b.double()), dict(activation="gelu"), dict(activation=1), dict(out=torch.empty_like(x).contiguous()), dict(out=x),
                dict(out=torch.empty_like(x, dtype=BF16)), dict(stats_out=torch.empty(2, 4, 1, device="cuda")), dict(eps=-1.0), dict(eps=float("nan")),
                dict(codes=True, out=torch.empty_like(x)), dict(codes="both", out=tc.Rows.empty(50, 16)), dict(codes=True, out=tc.Rows.empty(49, 16))):
        with pytest.raises((ValueError, TypeError, AttributeError, tc.TcError)):
            tc.tc_group_norm(ctx, x, 4, **bad)
    for args in ((x, y.contiguous(), stats), (x, y[:1], stats), (x, y.to(BF16), stats), (x, y, stats[:1]), (x, y, stats.double()), (x, y, torch.empty(2, 3, 2, device="cuda"))):
        with pytest.raises(ValueError):
            tc.tc_group_norm_backward(ctx, *args)
    wide = torch.zeros(1, 8200, 1, 1, device="cuda")
    with pytest.raises(tc.TcError, match="unsupported"):
        tc.tc_group_norm(ctx, wide, 8)
