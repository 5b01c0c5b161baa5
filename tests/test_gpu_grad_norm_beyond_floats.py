"""Gradients that are finite with a norm that is not a float: the norm reads infinity, the factor is finite, and the step is taken."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits", [32, 8])
def test_the_step_is_taken(bits):
    n, limit = 1000, 1e6
    g = [torch.full((n,), 3e38, device=DEV), torch.full((3,), -1.0, device=DEV)]
    p = [torch.zeros_like(x) for x in g]
    h = B.tbn_adamw_tensors(p, g, *B.tbn_adamw_state(p, bits))
    norm, scale = B.tbn_grad_norm(h, limit)
    length = math.sqrt(sum(x.double().square().sum().item() for x in g))
    assert math.isinf(norm.item()) and norm.item() > 0
    assert scale.item() == torch.tensor(limit / length, dtype=torch.float32).item() > 0
    B.tbn_adamw_step(h, 1, 1e-2, 0.9, 0.999, 1e-12, grad_scale=scale)
    # the first step is lr sign(g): m / bc1 = g and v / bc2 = g^2, a few dozen roundings of 2^-24
    assert ((p[0].double() + 1e-2).abs() <= 1e-2 * 40 * 2.0 ** -24).all()
    # 1e6 / 9.5e39 of a gradient of 1 is nothing next to eps
    assert (p[1].abs() <= 1e-2 * 1e-12).all()
