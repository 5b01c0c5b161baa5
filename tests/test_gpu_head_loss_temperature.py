"""Distillation at temperatures over the whole accepted range: every element against a 64-bit form with a bound of its own token and
class (tests/head_token_util.py)."""
import math

import pytest
import torch

from tests.head_token_util import DEV, check

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


def make(seed, T, d, V, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, d, generator=g) * scale).to(dtype).to(DEV)
    w = (torch.randn(V, d, generator=g) * (2.0 / math.sqrt(d)) * scale).to(dtype).to(DEV)
    dloss = ((0.5 + torch.rand(T, generator=g)) / T).to(DEV)
    return g, x, w, dloss, torch.randint(-1, V, (T,), generator=g).to(DEV)


@pytest.mark.parametrize("dtype,dloss_by_tau", [(torch.bfloat16, False), (torch.bfloat16, True), (torch.float32, False)])
@pytest.mark.parametrize("tau", [1e-30, 1e-12, 1e-3, 1e3, 1e12, 1e30])
def test_temperatures_at_both_ends(dtype, tau, dloss_by_tau):
    """Logits of the order of tau, so that the softmax is an ordinary one.  Where tau^2 leaves the range of fp32 so does the loss;
    gradients that leave it are infinities."""
    g, x, w, dloss, _ = make(8, 130, 64, 300, dtype, math.sqrt(tau))
    index = torch.randint(-1, 300, (130, 4), generator=g).to(DEV)
    logit = (torch.randn(130, 4, generator=g) * tau).to(DEV)
    names = ("lse", "dx", "dw", "db") + (("loss",) if 1e-18 < tau < 1e18 else ())
    got, _, _ = check(x, w, None, dloss / tau if dloss_by_tau else dloss, tau=tau, index=index, logit=logit, names=names)
    if tau < 1e-18:
        assert not bool(got["loss"].any())               # of order 1e-60


@BOTH
@pytest.mark.parametrize("tau", [1e-30, 1e-24, 1e-20])
def test_loss_near_temperature_zero(dtype, tau):
    """Logits of order 1: tau^2 is below fp32, tau^2 times a difference of logits / tau is not."""
    _, x, w, dloss, targets = make(9, 130, 64, 300, dtype)
    index = targets[:, None].clamp(min=0)
    got, _, _ = check(x, w, None, dloss, tau=tau, index=index, logit=torch.zeros(130, 1, device=DEV), names=("lse", "loss"))
    assert bool((got["loss"] > 0).any())
