"""Head losses with fp32 operands whose tokens, classes, features or sizes differ by many orders of magnitude: every element against
a 64-bit form with a bound of its own token and class (tests/head_token_util.py)."""
import math

import pytest
import torch

from tests.head_token_util import DEV, check

pytestmark = pytest.mark.gpu


def make(seed, T, d, V, scale_x=1.0, scale_w=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, d, generator=g) * scale_x).to(DEV)
    w = (torch.randn(V, d, generator=g) * (2.0 / math.sqrt(d)) * scale_w).to(DEV)
    dloss = ((0.5 + torch.rand(T, generator=g)) / T).to(DEV)
    return g, x, w, dloss, torch.randint(-1, V, (T,), generator=g).to(DEV)


@pytest.mark.parametrize("scale_x,scale_w", [(1e20, 1e-20), (1e-25, 1e25), (1e30, 1e-30), (1e-18, 1e-18), (1.0, 1.0)])
def test_fp32_operands_far_from_one(scale_x, scale_w):
    g, x, w, dloss, targets = make(1, 150, 80, 400, scale_x, scale_w)
    check(x, w, torch.randn(400, generator=g).to(DEV), dloss, targets=targets)


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e20, 1e30])
def test_fp32_loss_gradients_far_from_one(scale):
    _, x, w, dloss, targets = make(2, 150, 80, 400)
    check(x, w, None, dloss * scale, targets=targets)


@pytest.mark.parametrize("factor", [1e4, 1e6, 1e8, 1e10, 1e12])
def test_fp32_a_large_token_leaves_the_others_alone(factor):
    _, x, w, dloss, targets = make(3, 64, 512, 1000)
    x[17, 100] *= factor
    check(x, w, None, dloss, targets=targets)


def test_fp32_a_large_class_and_a_large_feature_leave_the_others_alone():
    _, x, w, dloss, targets = make(4, 90, 64, 300)
    w[33] *= 1e7
    bias = torch.zeros(300, device=DEV)
    bias[33] = -math.inf                                # a class that is masked out
    check(x, w, bias, dloss, targets=torch.where(targets == 33, torch.zeros_like(targets), targets), names=("lse", "loss", "db"))
    _, x, w, dloss, targets = make(5, 90, 64, 300)
    x[:, 7], w[:, 7] = 3.4e38, 0.0                      # rounding it up to bf16 would leave the range
    check(x, w, None, dloss * 1e-3, targets=targets)


def test_fp32_rare_classes_keep_their_gradient():
    """Classes of probability 1e-9 to 1e-30 that are nobody's target: their rows of dw are sums of nothing but such entries."""
    g, x, w, dloss, targets = make(6, 300, 64, 700)
    bias = torch.randn(700, generator=g).to(DEV)
    bias[400:500], bias[500:600], bias[600:] = -25.0, -50.0, -70.0
    got, val, _ = check(x, w, bias, dloss, targets=torch.where(targets >= 400, targets - 400, targets))
    for rows in (slice(400, 500), slice(500, 600), slice(600, 700)):
        rel = float((got["dw"][rows].double() - val["dw"][rows]).norm() / val["dw"][rows].norm())
        assert rel < 3e-5, (rows, rel)                   # the exponent: roundings of 2^-24 of 101 (bias), 131, 131 and twice 30 (lse), in log2


def test_fp32_rare_classes_in_distillation():
    g, x, w, dloss, _ = make(7, 200, 64, 500)
    bias = torch.randn(500, generator=g).to(DEV)
    bias[300:] = -40.0
    index = torch.randint(0, 300, (200, 6), generator=g).to(DEV)
    check(x, w, bias, dloss, tau=1.5, index=index, logit=torch.randn(200, 6, generator=g).to(DEV))


@pytest.mark.parametrize("every", [9, 1])
@pytest.mark.parametrize("factor", [1e3, 1e6, 1e9, 1e12])
@pytest.mark.parametrize("with_bias", [False, True])
def test_fp32_tokens_with_large_logits(every, factor, with_bias):
    """Alone or among ordinary ones, whose results they leave alone."""
    g, x, w, dloss, targets = make(10, 140, 64, 300)
    x[::every] *= factor
    got, _, _ = check(x, w, torch.randn(300, generator=g).to(DEV) if with_bias else None, dloss, targets=targets)
    assert all(bool(torch.isfinite(t).all()) for t in got.values())


@pytest.mark.parametrize("tau", [1e-30, 1e-12, 1e12, 1e30])
def test_fp32_temperatures_and_loss_gradients_at_both_ends(tau):
    g, x, w, dloss, _ = make(8, 130, 64, 300, math.sqrt(tau), math.sqrt(tau))
    index = torch.randint(-1, 300, (130, 4), generator=g).to(DEV)
    check(x, w, None, dloss / tau, tau=tau, index=index, logit=(torch.randn(130, 4, generator=g) * tau).to(DEV), names=("lse", "dx", "dw", "db"))
