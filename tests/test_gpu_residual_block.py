"""A residual block's gradients are those of the output it returned."""
import math

import pytest
import torch

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding

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


SHAPES = [(300, 256, 1, 1), (5, 192, 7, 7), (1, 64, 1, 1), (2, 320, 14, 14), (2000, 1024, 1, 1), (40, 130, 1, 1), (1, 3000, 5, 5)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_the_forward_pass_is_the_same_again(ctx, shape, dtype, monkeypatch):
    """The norm's gradient is asked for at the sum that the block returned and at the product behind it, bit for bit."""
    rand, c = _rand(1), shape[1]
    block = tc.ResidualBlock(ctx, rand(c, c) / math.sqrt(c), before=1 + 0.2 * rand(c), after=1 + 0.2 * rand(c), gate=0.5 * rand(c), scale=torch.full((1,), 0.8, device="cuda"))
    h, ds = rand(*shape).to(dtype), rand(*shape).to(dtype)
    products, at = [], []
    product, backward = tc.tc_matmul_blocks, tc.tc_residual_norms_backward
    monkeypatch.setattr(binding, "tc_matmul_blocks", lambda *a, **k: products.append(product(*a, **k)) or products[-1])
    monkeypatch.setattr(binding, "tc_residual_norms_backward", lambda ctx, s, y, *a, **k: at.append((s, y)) or backward(ctx, s, y, *a, **k))
    out = block(h)
    block.gradients(h, ds)
    (s, y), (inner, none) = at
    assert inner is h and none is None
    assert torch.equal(s, out)
    assert torch.equal(y, products[0]) and torch.equal(products[1], products[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES + [(20000, 64, 1, 1), (20, 48, 8, 8)])
def test_norms_as_tensor_and_codes_at_once(ctx, shape, dtype):
    rand, c = _rand(2), shape[1]
    h, y = rand(*shape).to(dtype), rand(*shape).to(dtype)
    for args in (dict(y=y, after=rand(c), gate=rand(c)), {}):
        args["before"] = rand(c)
        s, x = tc.tc_residual_norms(ctx, h, **args)
        _, codes = tc.tc_residual_norms(ctx, h, **args, blocks=True)
        s2, (x2, codes2) = tc.tc_residual_norms(ctx, h, **args, blocks="both")
        room = (torch.zeros_like(h), tc.Blocks.empty(codes.rows, c))
        s3, (x3, codes3) = tc.tc_residual_norms(ctx, h, **args, blocks="both", out=room)
        assert x3 is room[0] and codes3 is room[1]
        for a, b, q in ((s2, x2, codes2), (s3, x3, codes3)):
            assert torch.equal(a, s) and torch.equal(b, x)
            assert torch.equal(q.codes.view(torch.uint8)[:, :c], codes.codes.view(torch.uint8)[:, :c]) and torch.equal(q.scales[:, :q.rows], codes.scales[:, :q.rows])
    assert tc.tc_residual_norms(ctx, h, y, blocks="both")[1] is None
    for bad in (torch.zeros_like(h), (torch.zeros_like(h),), (None, torch.zeros_like(h)), (tc.Blocks.empty(codes.rows, c), torch.zeros_like(h))):
        with pytest.raises((ValueError, AttributeError)):
            tc.tc_residual_norms(ctx, h, before=rand(c), blocks="both", out=bad)
