"""The bf16 rounding of the gradient under a mean over the tokens that count: weights of 0 and 1 / n."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.head_token_util import DEV, reference, xent_teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [171, 300])
@pytest.mark.parametrize("zeros", [1, 20])
def test_a_mean_whose_first_tokens_weigh_nothing(T, zeros):
    """256 classes of one logit each: every q is 2^-8, so every dz / dloss is 2^-8 or 2^-8 - 1, which bf16 holds exactly.  With one
    weight for all tokens that have any, that leaves the sums' own error, (T / 16 + 8) cut-offs of 2^-23."""
    d, V = 64, 256
    g = torch.Generator().manual_seed(T)
    x, w = torch.randn(T, d, generator=g).bfloat16().to(DEV), torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    x[:, -1] = 0
    w[:, -1] = torch.randn(V, generator=g).bfloat16().to(DEV)
    targets = torch.randint(0, V, (T,), generator=g).to(DEV)
    dloss = torch.full((T,), 1.0 / T, device=DEV)
    dloss[:zeros] = 0
    _, lse = B.tbn_linear_xent_fwd(x, w, targets)
    dx, dw, _ = B.tbn_linear_xent_bwd(x, w, targets, lse, dloss, dw_dtype=B.F32)
    val, _ = reference(x, w, None, dloss, 1.0, xent_teacher(targets, V), B.F32)
    q = torch.full((T, V), 1.0 / V, dtype=torch.float64, device=DEV)
    q[torch.arange(T), targets] -= 1
    dz = (q * dloss.double()[:, None]).abs()
    assert bool(((dw.double() - val["dw"]).abs() <= dz.t() @ x.double().abs() * (T / 16 + 8) * 2.0 ** -23).all())
    assert bool(((dx.double() - val["dx"]).abs() <= dz @ w.double().abs() * (V / 16 + 8) * 2.0 ** -23 + val["dx"].abs() * 2.0 ** -8).all())
