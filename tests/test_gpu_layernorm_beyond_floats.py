"""Finite rows whose sum, or whose sum of squared deviations, is beyond the largest float: what the header says of them, and no other row."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [8, 33, 100, 501, 2048, 8187, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_beyond_floats(d, dtype):
    T = 41
    x = torch.randn(T, d, generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).to(dtype)
    gamma, beta = torch.full((d,), 1.5, device=DEV), torch.linspace(-1, 1, d, device=DEV)
    clean = B.tbn_layernorm_train_fwd(x, gamma, beta, y_dtype=B.F32)
    x[7] = 3e38                                                         # 8 of them are beyond 3.4e38
    x[20] = 0.0
    x[20, 0] = 2.0 ** 66                                                # a deviation of 7 / 8 of it and more: its square is 2^131
    y, _, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, y_dtype=B.F32)
    assert torch.isnan(y[7]).all() and not torch.isfinite(mean[7])
    assert rstd[20] == 0 and torch.equal(y[20], beta)
    others = [t for t in range(T) if t not in (7, 20)]
    assert torch.equal(y[others], clean[0][others]) and torch.equal(mean[others], clean[2][others]) and torch.equal(rstd[others], clean[3][others])
