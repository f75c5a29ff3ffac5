"""SiLU's derivative in the group norm's gradient, far from zero on both sides and whatever the value beside it."""
import pytest
import torch

import paper_1905_10830_b200 as tc

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


def _slope(z):
    s, r = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    return s * (1 + z * r), s, r


@pytest.mark.parametrize("beside", [0.0, 1.5, -20.0, -43.0, -44.0, -90.0, 90.0, 1e4])
@pytest.mark.parametrize("c", [4096, 4095])
@pytest.mark.parametrize("second", [False, True])
def test_slopes(ctx, beside, c, second):
    """Maps of two pixels, with a mean of 0 and a deviation of 1 as their statistics: z is x, and the bias's gradient the derivative at the pixel whose gradient is 1, the other's being 0."""
    far = torch.logspace(-3, 5, c // 2, dtype=torch.float64)
    z = torch.cat([-far, far, torch.zeros(c % 2, dtype=torch.float64)]).cuda().float()
    x, dy = torch.empty(1, 1, 2, c, device="cuda"), torch.zeros(1, 1, 2, c, device="cuda")
    at = 1 if second else 0
    x[0, 0, at], x[0, 0, 1 - at], dy[0, 0, at] = z, beside, 1.0
    stats = torch.tensor([0.0, 1.0], device="cuda").expand(1, c, 2).contiguous()
    one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    g = tc.tc_group_norm_backward(ctx, x.permute(0, 3, 1, 2), dy.permute(0, 3, 1, 2), stats, weight=one, bias=zero, activation="silu")
    z = z.double()
    want, s, r = _slope(z)
    # relative errors of e^-z (2 steps, and what its argument of |z| / ln 2 is rounded by), of s (the exponential's share r of it, the addition, the product, the reciprocal and the product with
    # the other's denominator: 4) and of r = e^-z s (both, and a product); the sum's and the last product's
    exponential = 2 + 1.5 * z.abs()
    of_s, of_r = r * exponential + 5, s * exponential + 6
    tol = STEP * (s * of_s * (1 + z.abs() * r) + s * z.abs() * r * of_r + 2 * s * (1 + z.abs() * r)) + torch.where(z < -43.5, 6e-18, 1e-37)
    off = (g.bias.double() - want).abs()
    assert (off <= tol).all(), (float((off / tol).max()), float(z[(off / tol).argmax()]))
    assert ((g.weight.double() - want * z).abs() <= tol * z.abs() + want.abs() * z.abs() * STEP + 1e-36).all()
