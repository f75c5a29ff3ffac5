"""Integer codes of maps of few channels, whose scales take as much memory as their values: images around the sizes that a block's shared memory holds."""
import pytest
import torch

import paper_1905_10830_b200 as tc
from tests.test_gpu_blocks import _matrix, _values
from tests.test_gpu_rows import _plain_codes, _same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(3, 1, 200, 200), (2, 1, 224, 224), (1, 1, 200, 200), (2, 2, 160, 160), (2, 2, 164, 168), (3, 3, 130, 140), (2, 1, 8, 4714), (2, 1, 8, 4715), (2, 1, 8, 4716),
                                   (2, 1, 1, 55296), (2, 1, 27, 1023), (2, 1, 201, 203)])
def test_codes_of_maps_of_few_channels(ctx, shape, dtype):
    x = _values(shape, sum(shape), dtype)
    for kind in ("pixels", "channels"):
        _same(tc.tc_quantize_rows(ctx, x, rows=kind), _plain_codes(_matrix(x, kind)))
    for kind, r in zip(("pixels", "channels"), tc.tc_quantize_rows(ctx, x, rows="both")):
        _same(r, _plain_codes(_matrix(x, kind)))
