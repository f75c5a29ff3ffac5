"""Residual norms (tc_residual_norms, its backward) against the formulas in 64 bits, their gradients by automatic and finite
differences, and a residual block of all the layer calls between two coded layers."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from synth import featuremaps as fm

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs(shape, dtype, gate, seed=1):
    g = _gen(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")                 # noqa: E731
    c = shape[1]
    wide = torch.exp(rand(c))[None, :, None, None]
    d = dict(h=(rand(*shape) * wide).to(dtype), y=(rand(*shape) * wide.flip(1) * 3).to(dtype), after=1 + 0.3 * rand(c), before=1 + 0.3 * rand(c),
             scale=torch.full((1,), 0.7, device="cuda"), gate=None)
    if gate == "channel":
        d["gate"] = rand(c)
    elif gate == "tensor":
        d["gate"] = rand(*shape).to(dtype)
    d["h"][0, :, 0, 0] = 0                  # a pixel of zeros on either side
    d["y"][-1, :, -1, -1] = 0
    return d


def _vec(v):
    return v.double()[None, :, None, None]


def _forward64(h, y, after, gate, scale, before, eps=EPS):
    s = h
    if y is not None:
        u = y
        if after is not None:
            u = y / torch.sqrt((y * y).mean(1, keepdim=True) + eps) * after
        if gate is not None:
            u = u * gate
        s = h + (u if scale is None else scale * u)
    return s, None if before is None else s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * before


def _in64(d):
    return dict(h=d["h"].double(), y=None if d["y"] is None else d["y"].double(), after=None if d["after"] is None else _vec(d["after"]),
                gate=None if d["gate"] is None else _vec(d["gate"]) if d["gate"].dim() == 1 else d["gate"].double(),
                scale=None if d["scale"] is None else d["scale"].double(), before=None if d["before"] is None else _vec(d["before"]))


def _chain(c):
    """Roundings of fp32 that a sum over c channels (at most c / 8 or 64 of them in a row, and the threads') and the factors behind it add up to."""
    return (c / 8 + 100) * 2.0 ** -24


SHAPES = [(1, 1, 1, 1), (1, 16, 1, 1), (3, 64, 1, 1), (1001, 64, 1, 1), (10007, 24, 1, 1), (77, 128, 1, 1), (5003, 104, 1, 1), (1, 4096, 1, 1), (3, 130, 1, 1), (300, 256, 1, 1), (17, 512, 1, 1), (9, 1000, 1, 1), (40, 1024, 1, 1), (5, 2048, 1, 1),
          (3, 2051, 1, 1), (2500, 400, 1, 1), (1900, 776, 1, 1), (1301, 2048, 1, 1), (700, 4096, 1, 1), (601, 4104, 1, 1), (2501, 301, 1, 1), (1303, 1021, 1, 1), (1201, 1538, 1, 1), (700, 4095, 1, 1), (603, 4130, 1, 1), (4, 8192, 1, 1), (2, 16384, 1, 1), (2, 9000, 1, 1), (3, 20, 7, 7), (2, 256, 14, 14), (1, 33, 5, 13), (2, 1000, 1, 33), (70, 16, 2, 2),
          (200, 48, 8, 8), (300, 100, 7, 7), (64, 500, 14, 14), (3, 1030, 6, 7), (1, 3000, 5, 5), (40, 264, 1, 30)]
MIXES = [("channel", ()), ("tensor", ()), ("none", ()), ("none", ("scale",)), ("channel", ("before",)), ("channel", ("after",)),
         ("none", ("after", "scale")), ("none", ("y", "after", "scale"))]


def _mix(shape, dtype, mix, seed=1):
    gate, without = mix
    d = _inputs(shape, dtype, gate, seed)
    for k in without:
        d[k] = None
    return d


def _check(got, want, tol, name):
    tol = tol + (want.abs() + tol) * torch.finfo(got.dtype).eps / 2 + 1e-37
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (name, int(bad.sum()), ((got.double() - want).abs() / tol).max().item())


def _check_forward(d, s, x):
    """s and x against the formulas; (x, its error but for the last rounding)."""
    s64, x64 = _forward64(**_in64(d))
    k = _chain(s64.shape[1])
    branch = (s64 - d["h"].double()).abs()
    # the sum: the branch's own roundings and one of the sum
    err_s = branch * k + s64.abs() * 2.0 ** -24
    if d["y"] is None:
        err_s = torch.zeros_like(s64)
    else:
        _check(s, s64, err_s, "s")
    if d["before"] is None:
        assert x is None
        return None, None
    # x: what the errors of s do to it (through itself and through the mean), and its own roundings
    r = 1 / torch.sqrt((s64 * s64).mean(1, keepdim=True) + EPS)
    b = _vec(d["before"]).abs()
    err_x = b * (err_s * r + s64.abs() * r ** 3 * (s64.abs() * err_s).mean(1, keepdim=True)) + x64.abs() * k
    _check(x, x64, err_x, "x")
    return x64, err_x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mix", MIXES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(ctx, shape, mix, dtype):
    d = _mix(shape, dtype, mix)
    keep = {k: None if v is None else v.clone() for k, v in d.items()}
    s, x = tc.tc_residual_norms(ctx, **d, eps=EPS)
    if d["y"] is None:
        assert s is d["h"]
    x64, err_x = _check_forward(d, s, x)
    if d["before"] is None:
        return
    s2, blocks = tc.tc_residual_norms(ctx, **d, eps=EPS, blocks=True)
    assert torch.equal(s, s2)
    want, err = (t.permute(0, 2, 3, 1).reshape(-1, shape[1]) for t in (x64, err_x))
    got = blocks.dequantize().double()
    scales = blocks.scales[:, :blocks.rows].double().t().repeat_interleave(128, 1)[:, :shape[1]]
    # the nearest e4m3 value: half a step of 2^-3 of the value, 2^-10 below the normal numbers; scale, reciprocal and product round too
    tol = torch.maximum(want.abs() * 2.0 ** -4, scales * 2.0 ** -10) * (1 + 1e-4) + err * 2
    assert ((got - want).abs() <= tol).all()
    amax = torch.stack([t.abs().amax(1) for t in want.split(128, 1)])
    err_max = torch.stack([t.amax(1) for t in err.split(128, 1)])
    assert ((blocks.scales[:, :blocks.rows].double() * 448 - amax.clamp_min(2.0 ** -100)).abs() <= err_max + amax * 2.0 ** -22 + 1e-33).all()
    for name, v in keep.items():
        assert v is None or torch.equal(v, d[name]), name


def _gradients64(d, dx, ds, s):
    """Gradients by automatic differentiation in 64 bits, the forward taken through the given (rounded) sum: with respect to y and
    the vectors at h = s - branch."""
    v = _in64(d)
    h = s.double()
    if v["y"] is not None:
        branch, _ = _forward64(torch.zeros_like(h), v["y"], v["after"], v["gate"], v["scale"], None)
        h = h - branch
    leaves = {"h": h}
    leaves.update({k: t for k, t in v.items() if k != "h" and t is not None})
    leaves = {k: t.clone().requires_grad_() for k, t in leaves.items()}
    s64, x64 = _forward64(leaves["h"], *[leaves.get(k) for k in ("y", "after", "gate", "scale", "before")])
    loss = (s64 * 0).sum()
    if x64 is not None:
        loss = loss + (x64 * dx.double()).sum()
    if ds is not None:
        loss = loss + (s64 * ds.double()).sum()
    grads = torch.autograd.grad(loss, list(leaves.values()), allow_unused=True)
    return {k: torch.zeros_like(t) if g is None else g for (k, t), g in zip(leaves.items(), grads)}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mix", MIXES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("with_ds", [True, False])
def test_backward(ctx, shape, mix, dtype, with_ds):
    d = _mix(shape, dtype, mix, 2)
    g = _gen(9)
    c = shape[1]
    pixels = shape[0] * shape[2] * shape[3]
    s = d["h"]
    dx = None if d["before"] is None else (torch.randn(shape, generator=g, device="cuda")).to(dtype)
    ds = (torch.randn(shape, generator=g, device="cuda")).to(dtype) if with_ds else None
    want = _gradients64(d, dx, ds, s)
    args = {k: d[k] for k in ("after", "gate", "scale", "before")}
    got = tc.tc_residual_norms_backward(ctx, s, d["y"], dx, ds, eps=EPS, **args)
    # Magnitudes: every sum with its terms' absolute values, so that cancellation is counted.
    k = 2 * _chain(c)
    v = _in64(d)
    s64 = s.double()
    size = torch.zeros_like(s64) if ds is None else ds.double().abs()
    zero = torch.zeros_like(s64)
    r = zero
    if dx is not None:
        r = 1 / torch.sqrt((s64 * s64).mean(1, keepdim=True) + EPS)
        t = (dx.double() * v["before"]).abs()
        size = size + r * t + s64.abs() * r ** 3 * (t * s64.abs()).mean(1, keepdim=True)
    _check(got.h, want["h"], size * k, "h")
    over_pixels = k + (96 + pixels / 128) * 2.0 ** -24      # a block's pixels in a row, the blocks' sums, the threads'
    vector = lambda t: t.sum((0, 2, 3))                     # noqa: E731
    if dx is not None:
        _check(got.before, want["before"].reshape(-1), vector((dx.double() * s64 * r).abs()) * over_pixels, "before")
    else:
        assert got.before is None
    if d["y"] is None:
        assert got.y is None and got.after is None and got.gate is None and got.scale is None
        return
    y = v["y"].abs()
    q = 1 / torch.sqrt((y * y).mean(1, keepdim=True) + EPS) if d["after"] is not None else torch.ones_like(y)
    n = y * q
    after = v["after"].abs() if d["after"] is not None else 1.0
    gate = v["gate"].abs() if d["gate"] is not None else 1.0
    scale = v["scale"] if d["scale"] is not None else 1.0
    dv = scale * size * gate * after
    size_y = q * (dv + n * (dv * n).mean(1, keepdim=True)) if d["after"] is not None else dv
    _check(got.y, want["y"], size_y * k, "y")
    if d["after"] is not None:
        _check(got.after, want["after"].reshape(-1), vector(scale * size * gate * n) * over_pixels, "after")
    if d["gate"] is not None:
        size_g = scale * size * after * n
        if d["gate"].dim() == 1:
            _check(got.gate, want["gate"].reshape(-1), vector(size_g) * over_pixels, "gate")
        else:
            _check(got.gate, want["gate"], size_g * k, "gate")
    if d["scale"] is not None:
        _check(got.scale, want["scale"], (size * gate * after * n).sum().reshape(1) * (over_pixels + c * 2.0 ** -24), "scale")
    again = tc.tc_residual_norms_backward(ctx, s, d["y"], dx, ds, eps=EPS, **args)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("shape", [(5, 200, 1, 1), (2, 24, 3, 3)])
def test_backward_against_differences(ctx, shape):
    """The loss' change along a direction in all inputs, by central differences in 64 bits, is the gradients' product with it."""
    d = _mix(shape, F32, ("channel", ()), 3)
    g = _gen(4)
    rand = lambda t: torch.randn(t.shape, generator=g, device="cuda")            # noqa: E731
    dx, ds = rand(d["h"]), rand(d["h"])
    s, _ = tc.tc_residual_norms(ctx, **d, eps=EPS)
    got = tc.tc_residual_norms_backward(ctx, s, d["y"], dx, ds, eps=EPS, **{k: d[k] for k in ("after", "gate", "scale", "before")})
    along = {k: rand(v) for k, v in d.items()}
    step = 1e-5

    def loss(sign):
        s64, x64 = _forward64(**_in64({k: v.double() + sign * step * along[k].double() for k, v in d.items()}))
        return (s64 * ds.double()).sum() + (x64 * dx.double()).sum()

    slope = (loss(1) - loss(-1)) / (2 * step)
    mine = sum((getattr(got, k).double() * along[k].double()).sum() for k in d)
    # the gradients are taken at the sum as it is stored (2^-24), in fp32; the difference's own error is of order step^2
    size = sum((getattr(got, k).double() * along[k].double()).abs().sum() for k in d)
    assert abs(mine - slope) <= size * (_chain(shape[1]) * 4 + 1e-8)


def test_views_at_odd_addresses_and_guards(ctx):
    for shape in ((7, 264, 1, 1), (3, 24, 3, 5)):
        for dtype in (F32, BF16):
            d = _mix(shape, dtype, ("tensor", ()), 5)
            n = math.prod(shape)

            def odd(t):
                flat = torch.full((t.numel() + 9,), 2.5, dtype=t.dtype, device="cuda")
                flat[1:1 + t.numel()] = t.reshape(-1)
                return flat, flat[1:1 + t.numel()].view(t.shape)

            rooms = {k: odd(v) for k, v in d.items()}
            room_s, s = odd(torch.zeros(shape, dtype=dtype, device="cuda"))
            room_x, x = odd(torch.zeros(shape, dtype=dtype, device="cuda"))
            got = tc.tc_residual_norms(ctx, **{k: v[1] for k, v in rooms.items()}, eps=EPS, sum_out=s, out=x)
            assert got[0] is s and got[1] is x
            _check_forward(d, s, x)                            # (another order of the sums than at aligned addresses: the same bounds)
            for room in (room_s, room_x):
                assert room[0] == 2.5 and (room[1 + n:] == 2.5).all()


def test_bad_values_stay_in_their_pixels(ctx):
    for shape in ((6, 300, 1, 1), (2, 40, 3, 3)):
        d = _mix(shape, F32, ("channel", ()), 6)
        d["h"][1, 2, 0, 0] = float("nan")
        d["y"][0, 3, -1, -1] = float("inf")
        s, x = tc.tc_residual_norms(ctx, **d, eps=EPS)
        bad = torch.zeros(shape[0], shape[2], shape[3], dtype=torch.bool, device="cuda")
        bad[1, 0, 0] = bad[0, -1, -1] = True
        assert torch.equal((~x.isfinite()).any(1), bad)
        assert torch.equal((~s.isfinite()).any(1), bad)
        _, b = tc.tc_residual_norms(ctx, **d, eps=EPS, blocks=True)
        assert torch.equal((~b.dequantize().isfinite()).any(1), bad.reshape(-1))


def test_no_pixels(ctx):
    e = lambda: torch.empty((0, 64, 1, 1), device="cuda")                         # noqa: E731
    d = dict(after=torch.ones(64, device="cuda"), gate=torch.ones(64, device="cuda"), scale=torch.ones(1, device="cuda"), before=torch.ones(64, device="cuda"))
    s, x = tc.tc_residual_norms(ctx, e(), e(), **d)
    assert s.shape == x.shape == (0, 64, 1, 1)
    g = tc.tc_residual_norms_backward(ctx, e(), e(), e(), e(), **d)
    for v in (g.after, g.gate, g.scale, g.before):
        assert not v.any()


def test_refusals(ctx):
    d = _mix((4, 64, 1, 1), F32, ("channel", ()), 7)
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms(ctx, d["h"])                                          # nothing to do
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms(ctx, d["h"], before=d["before"], gate=d["gate"])      # a gate of nothing
    with pytest.raises(ValueError):
        tc.tc_residual_norms(ctx, d["h"], d["y"][:3], after=d["after"])
    with pytest.raises(ValueError):
        tc.tc_residual_norms(ctx, d["h"], d["y"].to(BF16), after=d["after"])
    with pytest.raises(ValueError):
        tc.tc_residual_norms(ctx, d["h"], d["y"].cpu(), after=d["after"])
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms(ctx, d["h"], d["y"], after=d["after"], sum_out=d["h"])    # in place
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms(ctx, d["h"], d["y"], eps=-1.0)
    with pytest.raises(ValueError):
        tc.tc_residual_norms(ctx, d["h"], d["y"], after=d["after"][:-1])
    with pytest.raises(ValueError):
        tc.tc_residual_norms(ctx, d["h"], d["y"], after=d["after"].double())
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms(ctx, torch.zeros((1, 16400, 1, 1), device="cuda"), before=torch.ones(16400, device="cuda"))
    with pytest.raises(tc.TcError):
        tc.tc_residual_norms_backward(ctx, d["h"], d["y"], d["h"], d["y"], after=d["after"])     # dx without before


def _block(ctx, c, seed):
    g = _gen(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")                  # noqa: E731
    return dict(weight=rand(c, c) / math.sqrt(c), before=1 + 0.2 * rand(c), after=1 + 0.2 * rand(c), gate=0.5 * rand(c), scale=torch.full((1,), 0.8, device="cuda"))


@pytest.mark.parametrize("shape", [(300, 256, 1, 1), (5, 192, 7, 7), (1, 64, 1, 1), (2, 320, 14, 14)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_residual_block(ctx, shape, dtype):
    """The calls together, forward and gradients, against the same chain of plain operations in 64 bits on the codes that the
    calls make."""
    c = shape[1]
    v = _block(ctx, c, 8)
    block = tc.ResidualBlock(ctx, eps=EPS, **v)
    h = _inputs(shape, dtype, "none", 9)["h"]
    s = block(h)
    # operands: the same quantisation of the same x
    _, x_codes = tc.tc_residual_norms(ctx, h, before=v["before"], eps=EPS, blocks=True)
    y64 = (x_codes.dequantize().double() @ block.rows.dequantize().double().t()).reshape(shape[0], shape[2], shape[3], c).permute(0, 3, 1, 2)
    y = y64.to(dtype).double()                       # the block stores y in the maps' type
    s64, _ = _forward64(h.double(), y, _vec(v["after"]), _vec(v["gate"]), v["scale"].double(), None)
    # y may be off by a step of its type where it rounds to the other side, and with it the branch, through itself and the mean
    step = torch.finfo(dtype).eps + 1e-5
    branch = (s64 - h.double()).abs()
    scale_y = (v["scale"].double() * _vec(v["gate"]) * _vec(v["after"])).abs() / torch.sqrt((y * y).mean(1, keepdim=True) + EPS)
    slack = x_codes.dequantize().double().abs() @ block.rows.dequantize().double().abs().t()
    slack = slack.reshape(shape[0], shape[2], shape[3], c).permute(0, 3, 1, 2) * 2.0 ** -18
    _check(s, s64, branch * (2 * step + _chain(c)) + scale_y * slack * 2 + s64.abs() * 2.0 ** -24, "s")
    ds = torch.randn(shape, generator=_gen(10), device="cuda").to(dtype)
    g = block.gradients(h, ds)
    leaves = {k: t.double().requires_grad_() for k, t in (("h", h), *v.items())}
    x = leaves["h"] / torch.sqrt((leaves["h"] ** 2).mean(1, keepdim=True) + EPS) * leaves["before"][None, :, None, None]
    y = torch.einsum("nchw,oc->nohw", x, leaves["weight"])
    out, _ = _forward64(leaves["h"], y, leaves["after"][None, :, None, None], leaves["gate"][None, :, None, None], leaves["scale"], None)
    want = dict(zip(leaves, torch.autograd.grad((out * ds.double()).sum(), list(leaves.values()))))
    # A code is off by at most 2^-4 of its value, on average by about a third of that; a gradient holds three such operands (x, W, dy), whose
    # errors are independent: in the norm over all values sqrt(3) * 2^-4 / 2 at most where nothing cancels, twice that with the norms.
    # scale's is one sum over all values, ds gate u, which cancels: an error e of u moves it by at most |ds gate| |e| (Cauchy-Schwarz), and
    # |e| <= sqrt(2) * 2^-4 |u| with the two operands of the forward product, the norm's own part of it included.
    n64 = (y / torch.sqrt((y * y).mean(1, keepdim=True) + EPS) * leaves["after"][None, :, None, None]).detach()
    most = (ds.double() * _vec(v["gate"])).norm() * n64.norm() * math.sqrt(2) * 2.0 ** -4
    assert (g["scale"].double() - want.pop("scale")).abs() <= most
    for name, t in want.items():
        off = (g[name].double().reshape(t.shape) - t).norm()
        assert off <= math.sqrt(3) * 2.0 ** -4 * t.norm(), (name, (off / t.norm()).item())


def test_residual_blocks_between_coded_layers(ctx):
    """Residual blocks as stages of a chain of coded layers: calibrated one after the other, then run."""
    params = fm.layer_params(fm.LayerSpec(64, 14, 14, 0.9, None, 8100))
    cal, x = fm.make_maps(params, 24, calib=True, dtype=BF16).cuda(), fm.make_maps(params, 6, dtype=BF16).cuda()
    stages = [tc.ResidualBlock(ctx, **_block(ctx, 64, seed)) for seed in (1, 2)]
    layers = tc.calibrate_layer_by_layer(ctx, stages, cal, (6, 6), (False, False))
    maps, recons, bits = tc.run_chain(ctx, stages, layers, x)
    assert tc.tc_get_status(ctx) == 0
    assert torch.equal(maps[0], stages[0](x)) and torch.equal(maps[1], stages[1](recons[0]))
    for m, r, b in zip(maps, recons, bits):
        assert m.shape == r.shape == x.shape and 0 < b < m.numel() * 8
        # the quantiser's step bounds the distortion; the maps' own spread is far above it
        assert (m.float() - r.float()).square().mean() < 0.2 * m.float().var()


def test_captured_with_other_calls_between(ctx):
    shape = (50, 1000, 1, 1)
    d = _mix(shape, BF16, ("channel", ()), 12)
    dx = torch.randn(shape, generator=_gen(13), device="cuda").to(BF16)
    args = {k: d[k] for k in ("after", "gate", "scale", "before")}
    tc.tc_residual_norms_backward(ctx, d["h"], d["y"], dx, None, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s, x = tc.tc_residual_norms(ctx, d["h"], d["y"], **args)
        g = tc.tc_residual_norms_backward(ctx, s, d["y"], dx, None, **args)
    for seed in (14, 15):
        for k in ("h", "y"):
            d[k].copy_(torch.randn(shape, generator=_gen(seed), device="cuda"))
        tc.tc_residual_norms_backward(ctx, torch.randn(400, 2048, 1, 1, device="cuda"), None, torch.randn(400, 2048, 1, 1, device="cuda"), None,
                                      before=torch.ones(2048, device="cuda"))
        graph.replay()
        want_s, want_x = tc.tc_residual_norms(ctx, d["h"], d["y"], **args)
        want = tc.tc_residual_norms_backward(ctx, want_s, d["y"], dx, None, **args)
        assert torch.equal(s, want_s) and torch.equal(x, want_x)
        for a, b in zip(g, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(4_000_000, 16, 1, 1), (4_000_000, 20, 1, 1), (20_000, 1024, 1, 1), (1000, 16, 28, 28)])
def test_scale_gradient_of_many_pixels(ctx, shape):
    """Equal terms v = 1 + 0.45 * 2^-13, one a pixel (y = +-1 has the norm 1, ds is v in one channel): added one after the other in fp32, a chain of more than
    1024 of them loses nearly half of a unit in the last place each time."""
    n, c, h, w = shape
    pixels = n * h * w
    y = torch.ones(shape, device="cuda")
    y[:, 1::2] = -1
    ds = torch.zeros(shape, device="cuda")
    v = torch.tensor(1 + 0.45 * 2.0 ** -13, device="cuda")
    ds[:, 0] = v
    got = tc.tc_residual_norms_backward(ctx, y, y, None, ds, after=torch.ones(c, device="cuda"), scale=torch.ones(1, device="cuda"), eps=0.0)
    want = pixels * v.double()
    # A block's own sum carries its roundings: one (2^-24) where it leaves.  Of a warp's eight rows, or a lane's pixels: a sum over 32 lanes, 5 roundings, and one of two pixels.
    # Blocks: at most 592, by 32 lanes 19 in a row and 5 for the lanes'.  1 / sqrt(1) may be off by 2^-22 (twice: for y and in the pixel's part), the sum of 1 / c times c ones by 2^-23.
    tol = want * ((1 + 6 + 19 + 5) * 2.0 ** -24 + 2 * 2.0 ** -22 + 2.0 ** -23)
    assert (got.scale.double() - want).abs().item() <= tol.item(), ((got.scale.double() - want) / want).item()
