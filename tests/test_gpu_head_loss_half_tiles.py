"""Half tiles without rows: the pair's second CTA loads nothing for them, and its producer must not lose the pipeline's phase."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.head_token_util import DEV

pytestmark = pytest.mark.gpu


def test_backward_with_half_tiles_many_times():
    """38 tokens in the last tile of 256, many short tiles, several pieces of the vocabulary; the same bits and no wait that ran out,
    in each of 400 calls (one in 55 lost a phase)."""
    T, d, V = 8100, 128, 33001
    g = torch.Generator(device=DEV).manual_seed(T + d + V)
    x = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn(V, d, generator=g, device=DEV) * 0.17).to(torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    targets[torch.randperm(T, generator=g, device=DEV)[: T - 22 * 256 - 38]] = -100
    dloss = torch.full((T,), 1.0 / T, device=DEV)
    _, lse = B.tbn_linear_xent_fwd(x, w, targets)
    first = B.tbn_linear_xent_bwd(x, w, targets, lse, dloss)
    for _ in range(400):
        dx, dw, _ = B.tbn_linear_xent_bwd(x, w, targets, lse, dloss)
        assert B.tbn_last_device_status() == (0, 0)
    assert torch.equal(dx, first[0]) and torch.equal(dw, first[1])
