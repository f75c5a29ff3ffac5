"""A row's scale is its largest magnitude by 127, rounded once, whatever the significand."""
import pytest
import torch

import paper_1905_10830_b200 as tc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


@pytest.mark.parametrize("exponent", [1, -100, 0, 127, -37])
def test_scales_of_all_significands(ctx, exponent):
    bits = torch.arange(1 << 23, dtype=torch.int32, device="cuda") + ((exponent + 127) << 23)
    x = bits.view(torch.float32)
    r = tc.tc_quantize_rows(ctx, x.reshape(-1, 1, 1, 1))
    # (no quotient of a value by 127 lies halfway between two values of fp32, nor so near it that 64 bits do not tell: it differs from it by 1 / 254 of a step at least)
    assert torch.equal(r.scales, (x.double() / 127).float())
    assert (r.codes[:, 0] == 127).all()
