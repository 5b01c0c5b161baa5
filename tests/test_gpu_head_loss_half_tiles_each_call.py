"""Half tiles without rows, looked at in each call: the gradients against sums in 64 bits once, and the same bits ever after."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.head_token_util import DEV, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V,last", [(8100, 128, 33001, 38), (8100, 128, 33001, 1), (6000, 64, 20011, 128)])
def test_every_one_of_many_backward_calls(T, d, V, last):
    """`last` tokens in the last tile of 256, so that its second half has no rows."""
    g = torch.Generator(device=DEV).manual_seed(T + d + V + last)
    x = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn(V, d, generator=g, device=DEV) * 0.17).to(torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    kept = (T * 3 // 4) // 256 * 256 + last
    targets[torch.randperm(T, generator=g, device=DEV)[: T - kept]] = -100
    dloss = torch.full((T,), 1.0 / kept, device=DEV)
    first, _, _ = check(x, w, None, dloss, targets=targets)
    differ = torch.zeros(150, dtype=torch.bool, device=DEV)
    for i in range(len(differ)):
        dx, dw, _ = B.tbn_linear_xent_bwd(x, w, targets, first["lse"], dloss, dw_dtype=B.F32)
        differ[i] = (dx != first["dx"]).any() | (dw != first["dw"]).any()
        assert B.tbn_last_device_status() == (0, 0)
    assert not differ.any()
