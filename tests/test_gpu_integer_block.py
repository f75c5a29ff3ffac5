"""A residual block on 8-bit integers: norm, codes, product and sum together, its gradients, a chain of blocks whose gradients are clipped, and coded maps
around it."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from tests import plain_group_norm as plain

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _rand(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda")


def _block(ctx, c, groups, activation="relu"):
    r = _rand(1)
    weight, nw, nb = r(c, c) / math.sqrt(c), 1 + 0.2 * r(c), 0.2 * r(c)
    return tc.IntegerBlock(ctx, weight, groups=groups, norm_weight=nw, norm_bias=nb, activation=activation), weight, nw, nb


def _rows(t):
    return t.permute(0, 2, 3, 1).reshape(-1, t.shape[1]).double()


SHAPES = [((300, 256, 1, 1), 8), ((5, 192, 7, 7), 32), ((1, 64, 1, 1), 4), ((2, 320, 14, 14), 32), ((40, 130, 1, 1), 13), ((1, 96, 40, 40), 96)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_forward_is_within_the_codes_half_steps(ctx, shape, groups, last, dtype):
    block, weight, nw, nb = _block(ctx, shape[1], groups, "silu")
    h = _rand(2)(*shape).to(dtype)
    h = h.contiguous(memory_format=torch.channels_last) if last else h
    s = block(h)
    assert s.dtype == dtype and s.shape == h.shape and s.stride() == h.stride()
    x = _rows(plain.forward(h, groups, nw, nb, 1e-5, "silu")[0].reshape(shape))
    off_x = _rows(plain.forward_tolerance(h, groups, nw, nb, 1e-5, "silu").reshape(shape))
    w = weight.double()
    step = lambda m: m.abs().amax(1, keepdim=True) / 127                        # noqa: E731
    off_x = off_x + 0.5 * (step(x) + off_x.amax(1, keepdim=True) / 127) * (1 + 1e-6)
    off_w = 0.5 * step(w).expand_as(w) * (1 + 1e-6)
    y = x @ w.t()
    off = off_x @ w.abs().t() + (x.abs() + off_x) @ off_w.t() + y.abs() * 2.0 ** -21
    half = torch.finfo(dtype).eps / 2
    off = off + (y.abs() + off) * half                                          # y is rounded, and the sum
    want = _rows(h) + y
    assert ((_rows(s) - want).abs() <= off + (want.abs() + off) * half + 1e-30).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("shape,groups", [((64, 256, 1, 1), 8), ((5, 192, 7, 7), 32), ((3, 64, 20, 20), 4)])
def test_gradients(ctx, shape, groups, last, dtype):
    """Against autograd of the definition in 64 bits.  A code is off by up to half a step, evenly: amax / 127 / sqrt(12), which is 1.1 % of a row's rms where
    amax is 5 times that, for each operand; bf16 values in between by 2^-9 / sqrt(3), 0.1 %.  The products' two operands make 1.6 %, and the norm's
    gradient takes two directions out of what it is given: 4 % bounds it all, and 10 % each of the few values of a vector."""
    block, weight, nw, nb = _block(ctx, shape[1], groups, "silu")
    r = _rand(3)
    h, ds = r(*shape).to(dtype), r(*shape).to(dtype)
    if last:
        h, ds = (t.contiguous(memory_format=torch.channels_last) for t in (h, ds))
    g = block.gradients(h, ds)
    leaves = [t.double().requires_grad_() for t in (h, weight, nw, nb)]
    x, w, a, b = leaves
    v = x.reshape(shape[0], groups, -1)
    n = ((v - v.mean(2, keepdim=True)) / torch.sqrt(v.var(2, unbiased=False, keepdim=True) + 1e-5)).reshape(shape)
    y = torch.nn.functional.silu(n * a[:, None, None] + b[:, None, None])
    s = x + torch.einsum("oc,nchw->nohw", w, y)
    want = torch.autograd.grad((s * ds.double()).sum(), leaves)
    assert g["h"].dtype == dtype and g["h"].stride() == ds.stride() and g["weight"].dtype == F32
    for name, v in zip(("h", "weight", "norm_weight", "norm_bias"), want):
        off = float((g[name].double() - v).norm() / v.norm())
        assert off < (0.04 if name in ("h", "weight") else 0.1), (name, off)
    without = tc.IntegerBlock(ctx, weight, groups=groups).gradients(h, ds)
    assert without["norm_weight"] is None and without["norm_bias"] is None


def test_a_chain_is_clipped_together(ctx):
    c, r = 128, _rand(5)
    vec = lambda at: at + 0.2 * r(c)                                            # noqa: E731
    blocks = [_block(ctx, c, 8)[0], tc.ResidualBlock(ctx, r(c, c) / math.sqrt(c), before=vec(1), after=vec(1), gate=vec(0.5)), tc.IntegerBlock(ctx, r(c, c) / math.sqrt(c), groups=16)]
    h, ds = r(6, c, 7, 7).to(BF16), r(6, c, 7, 7).to(BF16)
    free, norm = tc.chain_gradients(ctx, blocks, h, ds, 1e9)
    values = [v for g in free for v in g.values() if v is not None]
    exact = math.sqrt(sum(float((v.double() ** 2).sum()) for v in values))
    assert [sorted(k for k, v in g.items() if v is not None) for g in free] == [["norm_bias", "norm_weight", "weight"], ["after", "before", "gate", "weight"], ["weight"]]
    assert abs(float(norm) / exact - 1) < 1e-6
    clipped, norm2 = tc.chain_gradients(ctx, blocks, h, ds, exact / 8)
    assert torch.equal(norm, norm2)                                             # the same bits again
    for a, b in zip((v for g in clipped for v in g.values() if v is not None), values):
        assert torch.allclose(a.double(), b.double() / 8, rtol=1e-6, atol=1e-30)


def test_between_coded_maps(ctx):
    c = 64
    block = _block(ctx, c, 8)[0]
    maps = _rand(1)(8, c, 14, 14).to(BF16)
    layers = tc.calibrate_layer_by_layer(ctx, [lambda t: t, block], maps, [6, 6], [False, False])
    coded, recons, bits = tc.run_chain(ctx, [lambda t: t, block], layers, maps)
    assert torch.equal(coded[1], block(recons[0])) and all(b > 0 for b in bits)
    for layer in layers:
        layer.close()


def test_a_captured_step(ctx):
    """Forward pass and gradients captured, replayed with other inputs, eager calls in between."""
    block = _block(ctx, 192, 32)[0]
    r = _rand(7)
    h, ds = r(5, 192, 7, 7).to(BF16), r(5, 192, 7, 7).to(BF16)
    block(h), block.gradients(h, ds)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        s, (g, norm) = block(h), tc.chain_gradients(ctx, [block, block], h, ds, 0.5)
    for turn in range(3):
        h.copy_(r(5, 192, 7, 7))
        ds.copy_(r(5, 192, 7, 7))
        want, (want_g, want_norm) = block(h), tc.chain_gradients(ctx, [block, block], h, ds, 0.5)
        graph.replay()
        block(r(9, 192, 14, 14).to(BF16))                                       # takes the context's memory
        torch.cuda.synchronize()
        assert torch.equal(s, want) and torch.equal(norm, want_norm)
        assert all(torch.equal(a[k], b[k]) for a, b in zip(g, want_g) for k in a)


def test_refusals(ctx):
    w = torch.randn(16, 16, device="cuda")
    for bad in (w[:8], w[0]):
        with pytest.raises(ValueError):
            tc.IntegerBlock(ctx, bad, groups=4)
    with pytest.raises(ValueError):
        tc.IntegerBlock(ctx, w, groups=3)(torch.randn(2, 16, 3, 3, device="cuda"))
