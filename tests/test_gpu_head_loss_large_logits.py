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
