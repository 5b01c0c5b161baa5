"""Rows of one value: their mean is that value, and what is left of them is nothing at all."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
VALUES = [1000.0, 3.0, -250.0, 96.0, 0.75]


@pytest.mark.parametrize("d", [1, 7, 25, 37, 49, 63, 96, 100, 300, 501, 768, 1000, 1500, 2047, 2056, 4097, 8184, 8185, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
def test_a_constant_row_is_its_mean(d, dtype, residual):
    """Multiples of 1/4 whose sums stay below 2^24 / 4 are added without a rounding, and a sum of n equal values over n is the value:
    every x - mean is 0, whatever 1 / sqrt(eps) it is multiplied by."""
    value = torch.tensor(VALUES, device=DEV).repeat(5)
    x = value[:, None].expand(-1, d).contiguous().to(dtype)
    other = torch.full_like(x, 0.25) if residual else None
    s = x if other is None else x + other
    gamma, beta = torch.full((d,), 7.0, device=DEV), torch.linspace(-1, 1, d, device=DEV)
    y, total, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, 1e-5, residual=other, y_dtype=B.F32)
    assert torch.equal(total, s) and torch.equal(mean, s[:, 0].float())
    assert ((rstd.double() * 1e-5 ** 0.5 - 1).abs() <= 2.0 ** -21).all()  # a rounded eps, its root, the rounding of the result
    assert torch.equal(y, beta.expand_as(y))
