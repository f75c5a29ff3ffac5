"""Group norms of so many maps that no run of pixels is shortened to keep the SMs busy: the longest sums a thread makes, of values of one sign whose roundings add up, of rows that begin at
16 bytes and others."""
import pytest
import torch

import paper_1905_10830_b200 as tc
from tests.test_gpu_group_norm import _check_backward, _check_forward, _vectors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,groups", [((300, 3, 128, 128), 1), ((200, 33, 56, 57), 33), ((100, 331, 28, 28), 1), ((300, 17, 40, 40), 17), ((64, 1032, 28, 28), 8), ((64, 516, 28, 28), 4), ((300, 8, 100, 100), 8),
                                          ((300, 130, 28, 28), 13)])
def test_long_sums_of_one_sign(ctx, shape, groups, dtype):
    n, c, h, w = shape
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (1 + 0.1 * torch.rand(n, h, w, c, generator=g, device="cuda")).to(dtype).permute(0, 3, 1, 2)
    dy = (1 + 0.001 * torch.rand(n, h, w, c, generator=g, device="cuda")).to(dtype).permute(0, 3, 1, 2)
    weight, bias = _vectors(c, 3)
    got = tc.tc_group_norm(ctx, x, groups, weight=weight, bias=bias)
    _check_forward(got, x, groups, weight, bias, 1e-5, None)
    _check_backward(tc.tc_group_norm_backward(ctx, x, dy, got[1], weight=weight, bias=bias), x, dy, got[1], groups, weight, bias, None)
