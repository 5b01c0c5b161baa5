"""Step numbers below 1 from the device count as 1, for the roundings of 8-bit states too; moments that keep nothing of the step before."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.test_gpu_adamw import DEV, F, H, check_step, clone, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("number", [0, -1, -2 ** 40])
def test_a_step_below_one_counts_as_one(bits, number):
    a = make([1000, 33], F, H, bits, seed=200, copy=True)
    b = clone(a)
    ha, hb = (B.tbn_adamw_tensors(**t, weight_decay=0.05) for t in (a, b))
    B.tbn_adamw_step(ha, 1, 1e-3, 0.9, 0.95, 1e-8, seed=11)
    B.tbn_adamw_step(hb, torch.tensor([number], device=DEV), 1e-3, 0.9, 0.95, 1e-8, seed=11)
    for k in a:
        assert all(x is None or torch.equal(x, y) for x, y in zip(a[k], b[k])), k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("b1,b2", [(0.0, 0.999), (0.9, 0.0), (0.0, 0.0)])
def test_betas_of_zero(bits, b1, b2):
    t = make([3000, 17], F, F, bits, seed=210)
    before = clone(t)
    args = (4, 1e-3, b1, b2, 1e-8)
    B.tbn_adamw_step(B.tbn_adamw_tensors(**t, weight_decay=0.1), *args, seed=5)
    for i in range(2):
        check_step(before, t, i, (*args, 0.1))
