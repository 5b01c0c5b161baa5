"""Head losses over vocabularies that the backward takes in several pieces, with contractions that are split, and with lists whose
table of starts is coarser than an epilogue warp's classes."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.head_token_util import DEV, check

pytestmark = pytest.mark.gpu


def make(seed, T, d, V, dtype, with_bias):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(T, d, generator=g, device=DEV).to(dtype)
    w = (torch.randn(V, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))).to(dtype)
    bias = torch.randn(V, generator=g, device=DEV) * 0.5 if with_bias else None
    return g, x, w, bias, (0.5 + torch.rand(T, generator=g, device=DEV)) / T


# several pieces of which the last is narrower, an odd vocabulary, part of the tokens left out.  d = 64 / 128: dX is split, its sums
# kept in slots from piece to piece; d = 20: fp32 and bf16 rows that are packed piece by piece
@pytest.mark.parametrize("dtype,T,d,V", [(torch.bfloat16, 8100, 64, 20011), (torch.bfloat16, 8100, 128, 33001), (torch.bfloat16, 16300, 20, 17011),
                                         (torch.float32, 4000, 64, 13001), (torch.float32, 4000, 256, 24001), (torch.float32, 8000, 21, 11003)])
@pytest.mark.parametrize("distill", [False, True])
def test_gradient_over_several_pieces(dtype, T, d, V, distill):
    g, x, w, bias, dloss = make(T + d + V, T, d, V, dtype, True)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    targets[torch.rand(T, generator=g, device=DEV) < 0.3] = -100
    if not distill:
        check(x, w, bias, dloss, targets=targets)
        return
    index = torch.randint(-1, V, (T, 7), generator=g, device=DEV)
    index[:, 3] = index[:, 5]                            # the same class twice
    index[targets < 0] = -1
    check(x, w, bias, dloss, tau=2.0, index=index, logit=torch.randn(T, 7, generator=g, device=DEV) * 3)


@pytest.mark.parametrize("dtype,T,V", [(torch.bfloat16, 7, 300_007), (torch.float32, 7, 150_001), (torch.bfloat16, 70, 540_001)])
@pytest.mark.parametrize("K", [3, 200])
def test_lists_over_more_classes_than_the_table_has_units(dtype, T, V, K):
    """Above 2046 units of an epilogue warp's classes the units are doubled, and a warp looks for its first entry from the unit's on."""
    g, x, w, bias, dloss = make(V + K, T, 16, V, dtype, False)
    index = torch.randint(0, V, (T, K), generator=g, device=DEV)
    index[::2, 1:] = (index[::2, :1] + torch.arange(1, K, device=DEV)) % V           # neighbours: many entries in one unit
    check(x, w, bias, dloss, tau=1.5, index=index, logit=torch.randn(T, K, generator=g, device=DEV) * 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_bad_token_in_the_backward(dtype):
    """A NaN and an infinity in kept rows: their rows of dx are NaN, every other row of dx is what it was."""
    g, x, w, _, dloss = make(3, 300, 64, 700, dtype, False)
    targets = torch.randint(0, 700, (300,), generator=g, device=DEV)
    run = lambda: B.tbn_linear_xent_bwd(x, w, targets, B.tbn_linear_xent_fwd(x, w, targets)[1], dloss)
    clean, _, _ = run()
    x[11, 3], x[150, 0] = math.nan, math.inf
    dx, dw, _ = run()
    bad = torch.zeros(300, dtype=torch.bool, device=DEV)
    bad[11], bad[150] = True, True
    assert bool(torch.isnan(dx[bad]).all()) and torch.equal(dx[~bad], clean[~bad])
    assert bool(torch.isnan(dw).any())
