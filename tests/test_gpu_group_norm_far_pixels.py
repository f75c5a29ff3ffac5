"""tc_group_norm of maps in which some pixels lie far from the rest: the first one (a padded or masked corner), first rows, the last, one in the middle."""
import pytest
import torch

import paper_1905_10830_b200 as tc
from tests.test_gpu_group_norm import _check_backward, _check_forward, _maps, _vectors

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


# On chip, one block and a cluster; runs through a ring, few and many of them; without one: rows not at 16 bytes, two channels a lane and one, more vectors than threads
SHAPES = [((1, 256, 14, 14), 32), ((2, 64, 40, 40), 64), ((3, 8, 100, 100), 1), ((300, 16, 56, 56), 4), ((40, 256, 28, 28), 256), ((1, 24, 700, 700), 3), ((40, 8, 128, 128), 8), ((3, 30, 60, 61), 3), ((200, 33, 56, 57), 33),
          ((60, 3, 200, 200), 1), ((2, 2056, 20, 21), 257), ((3, 4, 1, 3), 2),
          # blocks of a few dozen pixels
          ((290, 64, 7, 7), 64), ((30, 256, 14, 14), 256), ((100, 512, 5, 6), 512), ((1, 2048, 5, 5), 32), ((2, 33, 9, 9), 33)]


def _far(x, where, far):
    n, c, h, w = x.shape
    flat = x.permute(0, 2, 3, 1).reshape(n, h * w, c)         # (a copy where it is not a view)
    flat = flat.clone()
    at = {"first": slice(0, 1), "rows": slice(0, max(1, h // 16) * w), "last": slice(-1, None), "middle": slice(h * w // 2, h * w // 2 + 1)}[where]
    flat[:, at] = far.to(x.dtype)
    return flat.reshape(n, h, w, c).permute(0, 3, 1, 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("where", ["first", "rows", "last", "middle"])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_far_pixels(ctx, shape, groups, where, dtype):
    c = shape[1]
    spread = _maps(shape, 1, dtype).float().std((0, 2, 3))
    w, b = _vectors(c, 3)
    for deviations in (30.0, 100.0, 1000.0):
        x = _far(_maps(shape, 1, dtype), where, deviations * spread)
        got = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, eps=1e-5)
        _check_forward(got, x, groups, w, b, 1e-5, None)
    # means far from zero, and pixels that are zero
    x = _far(_maps(shape, 2, dtype, mean=0.0) + 300, where, torch.zeros(c, device="cuda"))
    got = tc.tc_group_norm(ctx, x, groups, weight=w, bias=b, eps=1e-5, activation="silu")
    _check_forward(got, x, groups, w, b, 1e-5, "silu")
    dy = _maps(shape, 7, dtype, 0.1)
    _check_backward(tc.tc_group_norm_backward(ctx, x, dy, got[1], weight=w, bias=b), x, dy, got[1], groups, w, b, None)


def test_the_same_pixel_everywhere_else(ctx):
    """Equal values but for the first pixel: mean and variance are known."""
    for n, c, h in ((1, 16, 14), (2, 8, 200), (2, 3, 200), (64, 64, 56)):
        x = _far(torch.full((n, h, h, c), 3.0, device="cuda").permute(0, 3, 1, 2), "first", torch.full((c,), 1003.0, device="cuda"))
        _, stats = tc.tc_group_norm(ctx, x, c, eps=0.0)
        p = 1.0 / (h * h)
        mean, rstd = 3.0 + 1000.0 * p, 1.0 / (1000.0 * (p * (1 - p)) ** 0.5)
        # some dozen roundings of quantities of the variance's size
        assert ((stats[:, :, 0].double() - mean).abs() <= 64 * 2.0 ** -24 * mean).all()
        assert ((stats[:, :, 1].double() / rstd - 1).abs() <= 64 * 2.0 ** -24).all()
