"""Head losses on logits so large that fp32 no longer resolves them to one: every element against a 64-bit form with a bound of its own
token and class (tests/head_token_util.py)."""
import math

import pytest
import torch

from tests.head_token_util import DEV, check

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


def make(seed, T, d, V, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).to(dtype).to(DEV)
    w = (torch.randn(V, d, generator=g) * (2.0 / math.sqrt(d))).to(dtype).to(DEV)
    dloss = ((0.5 + torch.rand(T, generator=g)) / T).to(DEV)
    return g, x, w, dloss, torch.randint(-1, V, (T,), generator=g).to(DEV)


@BOTH
@pytest.mark.parametrize("factor", [1e3, 1e6, 1e9, 1e12])
@pytest.mark.parametrize("T", [140, 300])               # rows read in place (bf16); rows packed
def test_loss_of_large_logits(dtype, factor, T):
    g, x, w, dloss, targets = make(10, T, 64, 300, dtype)
    x *= factor
    check(x, w, None, dloss, targets=targets, names=("lse", "loss"))
    check(x, w, torch.randn(300, generator=g).to(DEV) * factor, dloss, targets=targets, names=("lse", "loss"))


@BOTH
@pytest.mark.parametrize("tau", [1e-9, 1e-12, 1e-16])
def test_loss_of_a_cold_softmax(dtype, tau):
    """Logits of order 1 at a temperature near 0."""
    _, x, w, dloss, targets = make(9, 130, 64, 300, dtype)
    check(x, w, None, dloss, tau=tau, index=targets[:, None].clamp(min=0), logit=torch.zeros(130, 1, device=DEV), names=("lse", "loss"))


@pytest.mark.parametrize("every", [9, 1])
@pytest.mark.parametrize("factor", [1e3, 1e6, 1e9, 1e12])
@pytest.mark.parametrize("with_bias", [False, True])
def test_gradient_of_large_logits(every, factor, with_bias):
    """Tokens with large logits, alone or among ordinary ones."""
    g, x, w, dloss, targets = make(10, 140, 64, 300, torch.bfloat16)
    x[::every] *= factor
    got, _, _ = check(x, w, torch.randn(300, generator=g).to(DEV) if with_bias else None, dloss, targets=targets)
    assert all(bool(torch.isfinite(t).all()) for t in got.values())


@BOTH
@pytest.mark.parametrize("factor", [1e4, 1e7, 1e12])
def test_gradient_of_sure_tokens(dtype, factor):
    """Targets that are the largest logit by far: q is 1 there, the gradient 0 but for what is left of the rounding of lse."""
    _, x, w, dloss, _ = make(11, 140, 64, 300, dtype)
    x *= factor
    z = x.double() @ w.double().t()
    top = z.topk(2, 1).values
    targets = torch.where(top[:, 0] - top[:, 1] > 1e-3 * top[:, 0].abs(), z.argmax(1), torch.full((140,), -100, device=DEV))
    assert int((targets >= 0).sum()) > 70
    got, _, _ = check(x, w, None, dloss, targets=targets)
    size = float(dloss.max() * w.abs().max().float() * 2)
    # q >= exp(-2^-22 lse) below |log2 sum| = 4096, 1 above it
    assert float(got["dx"].float().abs().max()) <= size * 4096 * 2.0 ** -22
