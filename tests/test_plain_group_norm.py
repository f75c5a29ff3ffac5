"""The gradient formulas of the group norm that the kernels are tested with, against differences and against autograd of the definition."""
import pytest
import torch

from tests import plain_group_norm as plain


@pytest.mark.parametrize("kind", [None, "relu", "silu"])
@pytest.mark.parametrize("shape,groups", [((2, 6, 3, 4), 3), ((1, 4, 1, 1), 2), ((3, 5, 2, 2), 5), ((2, 8, 1, 3), 1)])
def test_gradients_are_those_of_differences(shape, groups, kind):
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)          # noqa: E731
    x, dy, w, b, eps = rand(*shape), rand(*shape), 1 + 0.3 * rand(shape[1]), rand(shape[1]), 1e-3
    loss = lambda x, w, b: (plain.forward(x, groups, w, b, eps, kind)[0] * plain.grouped(dy, groups)).sum()     # noqa: E731
    dx, dw, db = plain.backward(x, dy, groups, *plain.stats(x, groups, eps), w, b, kind)
    h = 1e-6
    for i, (t, grad) in enumerate(((x, dx.reshape(shape)), (w, dw), (b, db))):
        for _ in range(6):
            v = rand(*t.shape)
            at = lambda s: [u + s * h * v if j == i else u for j, u in enumerate((x, w, b))]     # noqa: E731
            assert abs(float((loss(*at(1)) - loss(*at(-1))) / (2 * h)) - float((grad * v).sum())) < 1e-5 * (1 + float((grad * v).abs().sum()))
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    for got, want in zip((dx.reshape(shape), dw, db), torch.autograd.grad(loss(*leaves), leaves)):
        assert torch.allclose(got, want, rtol=1e-9, atol=1e-11)
