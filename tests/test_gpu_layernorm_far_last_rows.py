"""Narrow rows share a warp, and some of them run out of rows before the others do: what is left of the last one adds nothing."""
import pytest
import torch

from tests.test_gpu_layernorm_far_rows import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [19_000, 19_003, 40_001])
@pytest.mark.parametrize("d", [31, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_a_warp_does_not_have(T, d, dtype):
    check(T, d, dtype, slice(None), True, False)
    check(T, d, dtype, slice(T // 2 - 50, None), False, True)
