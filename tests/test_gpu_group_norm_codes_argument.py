"""What tc_group_norm takes for `codes`."""
import pytest
import torch

import paper_1905_10830_b200 as tc

pytestmark = pytest.mark.gpu


def test_only_both_among_strings():
    ctx = tc.tc_create(0)
    x = torch.randn(2, 16, 5, 5, device="cuda").contiguous(memory_format=torch.channels_last)
    for bad in ("pixels", "channels", "", "true", "Both"):
        with pytest.raises(ValueError):
            tc.tc_group_norm(ctx, x, 4, codes=bad)
    assert isinstance(tc.tc_group_norm(ctx, x, 4, codes=True)[0], tc.Rows) and isinstance(tc.tc_group_norm(ctx, x, 4, codes=False)[0], torch.Tensor)
    y, rows = tc.tc_group_norm(ctx, x, 4, codes="both")[0]
    assert isinstance(y, torch.Tensor) and isinstance(rows, tc.Rows)
    ctx.close()
