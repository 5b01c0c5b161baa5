"""Embedding lookup (bit for bit) and its gradient (against sums in 64 bits).

A row of the gradient is a sum of n rows of dy in fp32, scaled: at most n + 2 roundings of 2^-24 of the sum of magnitudes, and the
rounding to dw's type; a row of one token is scaled and rounded, bit for bit."""
import math

import pytest
import torch

from oracle import tbn_oracle as O
from paper_2407_12075_b200 import binding as B
from paper_2407_12075_b200 import synth
from tests.util import to_dev

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": (torch.float32, B.F32), "bf16": (torch.bfloat16, B.BF16)}


def rand(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def some_ids(seed, T, V, kind):
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.rand(T, generator=g, device=DEV)
    ids = {"even": u, "skewed": u ** 6, "one": u * 0 + 0.37, "few": (u * 3).floor() / 3, "last": u * 0 + (V - 0.5) / V}[kind]
    ids = (ids * V).to(torch.int64).clamp_(0, V - 1)
    bad = torch.rand(T, generator=g, device=DEV)
    ids[bad < 0.04] = -1
    ids[(bad > 0.04) & (bad < 0.06)] = V
    ids[(bad > 0.06) & (bad < 0.08)] = -2 ** 62
    ids[(bad > 0.08) & (bad < 0.10)] = 2 ** 40 + 1
    return ids


@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 65536, 1024), (3, 10, 7), (50, 33, 255), (257, 1000, 256), (70, 500, 264), (1000, 77, 501), (33, 4000, 2056)])
@pytest.mark.parametrize("table_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
def test_lookup(T, V, d, table_dtype, y_dtype):
    table = rand(1, V, d, dtype=DT[table_dtype][0])
    ids = some_ids(2, T, V, "even")
    for scale, padding in ((1.0, -1), (math.sqrt(d), V // 2)):
        y = B.tbn_embedding_fwd(ids, table, scale, padding, DT[y_dtype][1])
        ok = (ids >= 0) & (ids < V) & (ids != padding)
        rows = table[torch.where(ok, ids, 0)].float() * torch.tensor(scale, dtype=torch.float32, device=DEV)
        assert torch.equal(y, torch.where(ok[:, None], rows, torch.zeros_like(rows)).to(DT[y_dtype][0]))
    assert B.tbn_embedding_fwd(ids.view(1, T, 1), table).shape == (1, T, 1, d)


@pytest.mark.parametrize("V,d,k", [(64, 256, 4), (100, 40, 8), (30, 7, 1), (30, 7, 5), (30, 7, 210), (33, 96, 11), (12, 501, 6), (10, 1030, 4), (16, 8, 16), (1000, 264, 3)])
@pytest.mark.parametrize("per_tile", [False, True])
@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
def test_tiled_lookup_reads_the_tiled_weight(V, d, k, per_tile, y_dtype):
    W = synth.normal(3, 1, V * d, 0.05)
    words, alphas = O.prepare(W, k, per_tile)
    tile, alpha = to_dev(words), to_dev(alphas)
    mode = B.ALPHA_PER_TILE if per_tile else B.ALPHA_PER_LAYER
    table = B.tbn_expand_tile(tile, V * d, k, alpha, mode).view(V, d)
    ids = torch.cat([torch.arange(V, device=DEV), some_ids(4, 60, V, "even")])
    for scale in (1.0, 2.5):
        y = B.tbn_embedding_tiled_fwd(ids, V, d, tile, k, alpha, mode, scale, -1, DT[y_dtype][1])
        assert torch.equal(y, B.tbn_embedding_fwd(ids, table, scale, -1, DT[y_dtype][1]))


def check_gradient(ids, dy, V, scale, padding, dw_dtype, before, got):
    d = dy.shape[1]
    ok = (ids >= 0) & (ids < V) & (ids != padding)
    at, rows = ids[ok], dy[ok].double()
    want = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, at, rows) * scale
    size = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, at, rows.abs()) * abs(scale)
    count = torch.bincount(at, minlength=V).double()[:, None]
    bound = (count + 2) * U * size
    if before is not None:
        want = want + before.double()
        bound += U * want.abs()
    bound += torch.finfo(dw_dtype).eps / 2 * 1.01 * want.abs() * (dw_dtype == torch.bfloat16) + 1e-40
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"{(err - bound).max().item()} over the bound"
    alone = (count[:, 0] == 0)
    assert torch.equal(got[alone], before[alone] if before is not None else torch.zeros_like(got[alone]))


GRADS = [(1, 1, 1), (6000, 40, 1021), (20000, 700, 333), (9, 3, 7), (40, 2, 2050), (7000, 900, 501), (8192, 300, 30), (8193, 70000, 24), (33, 5, 1003), (1, 70000, 64), (5, 3, 9), (40, 1000, 256), (300, 50, 257), (1024, 5000, 64), (1025, 1023, 40), (2049, 1024, 8), (4097, 65535, 72),
         (5000, 65536, 264), (9000, 200000, 33), (40000, 1500, 16), (140000, 3000, 8), (200000, 300000, 8)]


@pytest.mark.parametrize("T,V,d", GRADS)
@pytest.mark.parametrize("kind", ["even", "skewed", "one", "few", "last"])
def test_gradient(T, V, d, kind):
    i = GRADS.index((T, V, d))
    g_dtype, w_dtype = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")][(i + len(kind)) % 4]
    ids, dy = some_ids(5 + i, T, V, kind), rand(6, T, d, dtype=DT[g_dtype][0])
    scale, padding = (1.0, -1) if i % 2 else (math.sqrt(d), int(ids[T // 2]))
    got = B.tbn_embedding_bwd(ids, dy, V, scale, padding, DT[w_dtype][1])
    check_gradient(ids, dy, V, torch.tensor(scale, dtype=torch.float32).item(), padding, DT[w_dtype][0], None, got)
    assert torch.equal(got, B.tbn_embedding_bwd(ids, dy, V, scale, padding, DT[w_dtype][1]))
    before = rand(7, V, d, dtype=DT[w_dtype][0])
    added = B.tbn_embedding_bwd(ids, dy, V, scale, padding, add_to=before.clone())
    check_gradient(ids, dy, V, torch.tensor(scale, dtype=torch.float32).item(), padding, DT[w_dtype][0], before, added)


def test_ids_of_three_digits_and_more():
    """Vocabularies beyond 2^20 are sorted in three passes; the gradient of a narrow table stays small."""
    for V in (2 ** 20 - 1, 2 ** 20, 5 * 10 ** 6, 2 ** 27 + 3):
        ids, dy = some_ids(8, 3000, V, "even"), rand(9, 3000, 2)
        ids[::3] = ids[0].clamp(0, V - 1)
        got = B.tbn_embedding_bwd(ids, dy, V)
        check_gradient(ids, dy, V, 1.0, -1, torch.float32, None, got)
        del got
        torch.cuda.empty_cache()


def test_gradient_against_differences():
    """sum(y * g) moves by scale times the sum of g over the tokens of a row: the lookup is linear, so one difference is exact up to roundings."""
    T, V, d = 60, 9, 5
    table, ids, dy = rand(10, V, d), some_ids(11, T, V, "even"), rand(12, T, d)
    dw = B.tbn_embedding_bwd(ids, dy, V, 1.5)
    for v in range(V):
        moved = table.clone()
        moved[v, v % d] += 1.0
        change = ((B.tbn_embedding_fwd(ids, moved, 1.5) - B.tbn_embedding_fwd(ids, table, 1.5)).double() * dy.double()).sum().item()
        assert abs(change - dw[v, v % d].item()) < 60 * 1e-5


def test_no_token_and_no_valid_token():
    for ids in (torch.empty(0, dtype=torch.int64, device=DEV), torch.full((70,), -1, device=DEV), torch.full((3000,), 4, device=DEV)):
        dy = torch.full((len(ids), 24), float("nan"), device=DEV)        # nothing of a row that is left out reaches the result
        dw = B.tbn_embedding_bwd(ids, dy, 10, padding_idx=4)
        assert dw.shape == (10, 24) and not dw.any()
        before = rand(13, 10, 24)
        assert torch.equal(B.tbn_embedding_bwd(ids, dy, 10, padding_idx=4, add_to=before.clone()), before)
        assert not B.tbn_embedding_fwd(ids, torch.full((10, 24), float("inf"), device=DEV), padding_idx=4).any()


def test_tables_beyond_32_bit_offsets():
    V, d = 66001, 32776                                                  # 2.16e9 elements
    ids = torch.tensor([0, V - 1, 12345, V - 1, 65999, 3], device=DEV)
    table = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    for v in (0, 3, 12345, 65999, V - 1):
        table[v] = v % 100 + 1
    y = B.tbn_embedding_fwd(ids, table)
    assert torch.equal(y, table[ids])
    dw = B.tbn_embedding_bwd(ids, y, V)
    assert torch.equal(dw[V - 1], 2 * table[V - 1]) and torch.equal(dw[65999], table[65999])
    assert int((dw != 0).any(1).sum()) == 5
    assert torch.equal(B.tbn_embedding_bwd(ids, y, V, add_to=dw)[V - 1], 4 * table[V - 1])


@pytest.mark.parametrize("T,V,d,add", [(700, 90, 33, False), (5000, 300, 64, True)])
def test_workspace_contents_and_surroundings(T, V, d, add):
    ids, dy = some_ids(14, T, V, "skewed"), rand(15, T, d)
    need, pad = B.tbn_embedding_bwd_workspace_bytes(T, d, V), 1024
    outs = []
    for fill in (0, 255):
        ws = torch.full((need + 2 * pad,), fill, dtype=torch.uint8, device=DEV)
        dw = torch.full((V * d + 128,), 0.5, device=DEV)
        assert B.lib().tbn_embedding_bwd(ids.data_ptr(), T, dy.data_ptr(), B.F32, V, d, -1, 1.0, dw.data_ptr() + 256, B.F32, int(add), ws.data_ptr() + pad,
                                         need, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert (ws[:pad] == fill).all() and (ws[need + pad:] == fill).all() and (dw[:64] == 0.5).all() and (dw[-64:] == 0.5).all()
        outs.append(dw)
    assert torch.equal(*outs)
    check_gradient(ids, dy, V, 1.0, -1, torch.float32, torch.full((V, d), 0.5, device=DEV) if add else None, outs[0][64:-64].view(V, d))


def test_two_streams_at_once():
    jobs = []
    for i in range(2):
        ids, dy = some_ids(16 + i, 20000, 4000, "skewed"), rand(18 + i, 20000, 128)
        jobs.append((ids, dy, B.tbn_embedding_bwd(ids, dy, 4000)))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in jobs], []
    for _ in range(4):
        for (ids, dy, _), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                outs.append(B.tbn_embedding_bwd(ids, dy, 4000))
    torch.cuda.synchronize()
    assert all(torch.equal(o, jobs[i % 2][2]) for i, o in enumerate(outs))
