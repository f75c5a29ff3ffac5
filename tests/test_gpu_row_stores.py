"""Products of short sums whose rows leave by asynchronous copies: columns behind the last whole tile and warps behind the last row, several times over, bit for
bit."""
import pytest
import torch

import paper_1905_10830_b200 as tc
from tests.test_gpu_rows import _operand, _want

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = tc.tc_create(0)
    yield c
    assert tc.tc_get_status(c) == 0
    c.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [4, 8, 32, 36, 40, 64, 96, 128, 132, 136, 160, 192, 224])
def test_products_of_short_sums(ctx, rest, dtype):
    for n, k, o in ((25088, 320, 768 + rest), (8200, 512, 1024 + rest), (20010, 64, 256 + rest)):
        a, b = _operand(n, k, 1), _operand(o, k, 2)
        bias = torch.randn(o, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
        want = _want(a, b, bias, False, dtype, (n, 1, 1))
        for _ in range(8):
            assert torch.equal(tc.tc_matmul_rows(ctx, a, b, dtype=dtype, bias=bias), want)
