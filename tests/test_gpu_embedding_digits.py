"""The embedding's gradient over vocabularies whose ids are sorted by two, three and four digits: more tokens than one launch ranks."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.test_gpu_embedding import DT, U, rand, some_ids

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(ids, dy, V, scale, before, got):
    """Rows that a token names against sums in 64 bits, all others against what they were; of a large table only those are widened."""
    ok = (ids >= 0) & (ids < V)
    seen, place = ids[ok].unique(return_inverse=True)
    rows = dy[ok].double()
    zeros = torch.zeros(len(seen), dy.shape[1], dtype=torch.float64, device=DEV)
    want, size = zeros.index_add(0, place, rows) * scale, zeros.index_add(0, place, rows.abs()) * abs(scale)
    count = torch.bincount(place, minlength=len(seen)).double()[:, None]
    bound = (count + 2) * U * size
    if before is not None:
        want += before[seen].double()
        bound += U * want.abs()
    bound += torch.finfo(got.dtype).eps / 2 * 1.01 * want.abs() * (got.dtype == torch.bfloat16) + 1e-40
    assert ((got[seen].double() - want).abs() <= bound).all()
    rest = got.clone()
    rest[seen] = 0 if before is None else before[seen]
    assert not rest.any() if before is None else torch.equal(rest, before)


@pytest.mark.parametrize("V,d", [(2 ** 20 - 1, 24), (2 ** 20, 24), (2 ** 20 + 5, 33), (5_000_000, 9), (2 ** 27 + 3, 2), (2 ** 30 - 1, 1), (2 ** 30 + 7, 1)])
@pytest.mark.parametrize("T", [8193, 30_001, 150_000])
@pytest.mark.parametrize("kind", ["even", "skewed", "few"])
def test_gradient_over_large_vocabularies(V, d, T, kind):
    ids, dy = some_ids(21, T, V, kind), rand(22, T, d, dtype=DT["bf16"][0])
    ids[::3] = (ids[::3] * 7919).remainder(V)                           # differences in the lowest digits too
    ids[5::11] = ids[5]
    got = B.tbn_embedding_bwd(ids, dy, V, 1.5, dw_dtype=B.BF16)
    check(ids, dy, V, 1.5, None, got)
    assert torch.equal(got, B.tbn_embedding_bwd(ids, dy, V, 1.5, dw_dtype=B.BF16))
    before = rand(23, 1000, d, dtype=DT["bf16"][0])[torch.arange(V, device=DEV) % 1000] if V <= 5_000_000 else torch.full_like(got, 0.5)
    check(ids, dy, V, 1.5, before, B.tbn_embedding_bwd(ids, dy, V, 1.5, add_to=before.clone()))
