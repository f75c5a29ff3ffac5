"""Gradients of the residual norms (tc_residual_norms_backward) at the ends of what the call takes -- no eps, tiles of maps that the last pixels
fill in part, values far from 1, tensors at any address -- against the closed form in 64 bits."""
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


def _inputs(shape, dtype, gate, before, seed, size=1.0, with_ds=True):
    """Arguments of the call; values of order `size`, none of them zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")                 # noqa: E731
    values = lambda: rand(*shape) + torch.where(rand(*shape) < 0, -0.2, 0.2)      # noqa: E731
    c = shape[1]
    d = dict(s=(values() * size).to(dtype), y=(values() * size).to(dtype), dx=values().to(dtype) if before else None, ds=values().to(dtype) if with_ds else None,
             after=1 + 0.3 * rand(c), gate=None, scale=torch.full((1,), 0.7, device="cuda"), before=1 + 0.3 * rand(c) if before else None)
    if gate != "none":
        d["gate"] = values().to(dtype) if gate == "tensor" else rand(c)
    return d


def _close(got, want, tol, name):
    # half a step of the type where the result is rounded, its smallest one where that is more
    tol = tol + (want.abs() + tol) * torch.finfo(got.dtype).eps / 2 + 2.0 ** -133
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (name, int(bad.sum()), ((got.double() - want).abs() / tol).max().item())


def _check(d, got, eps):
    """Every gradient against its formula; bounds from the sums of the terms' magnitudes, with a rounding for each addition in a row (c / 8 channels at
    most, and the threads'; of the pixels a block's, the blocks', the threads')."""
    s, y = d["s"].double(), d["y"].double()
    c = s.shape[1]
    pixels = s.shape[0] * s.shape[2] * s.shape[3]
    vec = lambda v: v.double()[None, :, None, None]                              # noqa: E731
    mean = lambda t: t.mean(1, keepdim=True)                                     # noqa: E731
    total = lambda t: t.sum((0, 2, 3))                                           # noqa: E731
    after, scale = vec(d["after"]), d["scale"].double()
    gate = torch.ones((), dtype=torch.float64, device="cuda") if d["gate"] is None else vec(d["gate"]) if d["gate"].dim() == 1 else d["gate"].double()
    k = 2 * (c / 8 + 100) * 2.0 ** -24
    over = k + (96 + pixels / 128) * 2.0 ** -24
    big_d, size = torch.zeros_like(s), torch.zeros_like(s)
    if d["ds"] is not None:
        big_d, size = d["ds"].double(), d["ds"].double().abs()
    if d["before"] is not None:
        r = 1 / torch.sqrt(mean(s * s) + eps)
        t = d["dx"].double() * vec(d["before"])
        big_d = big_d + r * t - (s * r) * (r * mean(t * (s * r)))
        size = size + r * t.abs() + (s * r).abs() * (r * mean((t * (s * r)).abs()))
        n = d["dx"].double() * (s * r)
        _close(got.before, total(n), total(n.abs()) * over, "before")
    else:
        assert got.before is None
    _close(got.h, big_d, size * k, "h")
    q = 1 / torch.sqrt(mean(y * y) + eps)
    n = y * q
    v, size_v = scale * big_d * gate * after, scale * size * (gate * after).abs()
    _close(got.y, q * (v - n * mean(v * n)), q * (size_v + n.abs() * mean(size_v * n.abs())) * k, "y")
    _close(got.after, total(scale * big_d * gate * n), total(scale * size * (gate * n).abs()) * over, "after")
    of_gate, size_gate = scale * big_d * after * n, scale * size * (after * n).abs()
    if d["gate"] is None:
        assert got.gate is None
    elif d["gate"].dim() == 1:
        _close(got.gate, total(of_gate), total(size_gate) * over, "gate")
    else:
        _close(got.gate, of_gate, size_gate * k, "gate")
    _close(got.scale, (big_d * gate * after * n).sum().reshape(1), (size * (gate * after * n).abs()).sum().reshape(1) * (over + c * 2.0 ** -24), "scale")


def _run(ctx, d, eps):
    return tc.tc_residual_norms_backward(ctx, d["s"], d["y"], d["dx"], d["ds"], eps=eps, **{k: d[k] for k in ("after", "gate", "scale", "before")})


# 37 * 196 pixels leave 20 of 32 or 4 of 16 in the last tile, 3 * 49 leave 19, 3 and 3 (odd: a lane with one pixel), 1 * 65 one of 64, 1 * 33 one; more channels than a tile
# holds take the kernel without one; rows of 64 and 200 channels share warps and blocks
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(37, 64, 14, 14), (37, 256, 14, 14), (3, 24, 7, 7), (3, 264, 7, 7), (200, 520, 7, 7), (1, 20, 5, 13), (1, 1000, 1, 33), (1, 3000, 5, 5), (301, 64, 1, 1),
                                   (301, 200, 1, 1)])
@pytest.mark.parametrize("gate", ["channel", "tensor"])
@pytest.mark.parametrize("before", [True, False])
@pytest.mark.parametrize("eps", [0.0, 1e-28])
def test_without_eps(ctx, shape, dtype, gate, before, eps):
    d = _inputs(shape, dtype, gate, before, 3)
    _check(d, _run(ctx, d, eps), eps)


# The forward takes such values exactly (their squares and the sum over 64 to 520 channels stay within fp32), and so do the gradients.  1e17: r^2 times
# a gradient of 1e-6 and less is subnormal.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(37, 64, 14, 14), (40, 264, 7, 7), (1, 3000, 5, 5), (301, 64, 1, 1), (301, 201, 1, 1), (2500, 520, 1, 1), (2500, 521, 1, 1)])
@pytest.mark.parametrize("gate", ["none", "channel", "tensor"])
@pytest.mark.parametrize("size,eps", [(1e12, 1e-6), (1e15, 1e-6), (1e17, 0.0), (1e-14, 0.0), (1e-17, 0.0)])
@pytest.mark.parametrize("with_ds", [True, False])
def test_values_far_from_one(ctx, shape, dtype, gate, size, eps, with_ds):
    d = _inputs(shape, dtype, gate, True, 4, size, with_ds)
    if gate == "tensor":
        d["gate"] = _inputs(shape, dtype, gate, True, 5)["s"]
    d["dx"] = (d["dx"].float() * 1e-3).to(dtype)
    _check(d, _run(ctx, d, eps), eps)
