"""The widest rows, tiles of more than 2^32 bits, and a token list of a billion and a half."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.test_gpu_embedding import check_gradient, rand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [2 ** 23, 2 ** 23 - 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_widest_rows(d, dtype):
    V = 3
    ids = torch.tensor([2, 0, 2, -1, 2, 2, 2, 2, 2, 2, 0, 2, 3], device=DEV)          # the run of 2 goes on in a second piece
    table, dy = rand(400, V, d, dtype=dtype), rand(401, len(ids), d, dtype=dtype)
    y = B.tbn_embedding_fwd(ids, table, 2.0)
    ok = (ids >= 0) & (ids < V)
    assert torch.equal(y[ok], table[ids[ok]] * 2) and not y[~ok].any()
    del y
    check_gradient(ids, dy, V, 0.5, -1, dtype, None, B.tbn_embedding_bwd(ids, dy, V, 0.5))
    before = rand(402, V, d, dtype=dtype)
    check_gradient(ids, dy, V, 0.5, -1, dtype, before, B.tbn_embedding_bwd(ids, dy, V, 0.5, add_to=before.clone()))


@pytest.mark.parametrize("V,d,k", [(2 ** 21 + 8, 4096, 1), (2 ** 22 + 16, 4104, 4), (2 ** 21 + 8, 2049, 1), (2 ** 23 - 2, 1025, 2)])
def test_tiles_beyond_32_bit_offsets(V, d, k):
    q = V * d // k
    g = torch.Generator(device=DEV).manual_seed(V + d)
    words = -(-q // 128) * 4
    tile = torch.randint(-2 ** 31, 2 ** 31, (words,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    keep = (q - torch.arange(words, device=DEV) * 32).clamp_(0, 32)
    tile &= ((torch.ones_like(keep) << keep) - 1).to(torch.int32)
    alpha = 0.5 + torch.rand(k, generator=g, device=DEV)
    ids = torch.randint(0, V, (500,), generator=g, device=DEV)
    ids[:6] = torch.tensor([0, V - 1, V // k - 1, V // k, q // d, V - 2], device=DEV).clamp(0, V - 1)
    y = B.tbn_embedding_tiled_fwd(ids, V, d, tile, k, alpha, B.ALPHA_PER_TILE, 3.0, y_dtype=B.F32)
    f = ids[:, None] * d + torch.arange(d, device=DEV)
    bit = (tile[(f % q) >> 5] >> (f % q & 31).to(torch.int32)) & 1
    assert torch.equal(y, (2 * bit - 1).float() * (alpha * 3.0)[f // q])


def test_many_tokens():
    """Every sum of ones is a whole number below 2^24."""
    T, V = 1_500_000_001, 1021
    ids = torch.randint(-3, V + 3, (T,), generator=torch.Generator(device=DEV).manual_seed(410), device=DEV)
    dw = B.tbn_embedding_bwd(ids, torch.ones(T, 1, dtype=torch.bfloat16, device=DEV), V, dw_dtype=B.F32)
    want = torch.zeros(V + 6, dtype=torch.int64, device=DEV)
    for part in ids.split(1 << 28):
        want += torch.bincount(part + 3, minlength=V + 6)
    assert torch.equal(dw[:, 0].long(), want[3:V + 3])
    table = torch.arange(1, V + 1, dtype=torch.float32, device=DEV).view(V, 1)
    y = B.tbn_embedding_fwd(ids, table, y_dtype=B.F32)
    for rows, part in zip(y.split(1 << 28), ids.split(1 << 28)):
        assert torch.equal(rows[:, 0], torch.where((part >= 0) & (part < V), part + 1, 0).float())
    del y, ids, dw
    torch.cuda.empty_cache()
