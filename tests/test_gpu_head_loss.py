"""GPU parity of the head losses (cross entropy and distillation, forward and backward) against plain 64-bit forms, with
element-wise bounds derived from the roundings that take place (tests/head_util.py)."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.head_util import assert_within, bounds, reference, teacher_matrix
from tests.util import DEV

pytestmark = pytest.mark.gpu


def make(seed, T, d, V, dtype, with_bias, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).to(dtype)
    w = (torch.randn(V, d, generator=g) * (scale / math.sqrt(d))).to(dtype)
    bias = torch.randn(V, generator=g) * 0.5 if with_bias else None
    dloss = (0.5 + torch.rand(T, generator=g)) / max(T, 1)
    return g, x, w, bias, dloss


def one_hot(targets, V, ignore=-100):
    T = targets.shape[0]
    dense = torch.zeros(T, V, dtype=torch.float64)
    some = (targets != ignore) & (targets >= 0) & (targets < V)
    dense[some.nonzero()[:, 0], targets[some]] = 1.0
    return dense, torch.zeros(T, dtype=torch.float64), some


def on_gpu(*ts):
    return [t.to(DEV) if t is not None else None for t in ts]


def check_xent(x, w, bias, targets, dloss, dw_dtype=None, ignore=-100):
    ref = reference(x, w, bias, dloss, 1.0, *one_hot(targets, w.shape[0], ignore))
    code = (B.F32 if x.dtype == torch.float32 else B.BF16) if dw_dtype is None else dw_dtype
    bd = bounds(ref, x, w, 1.0, code)
    X, W, b, t, g = on_gpu(x, w, bias, targets, dloss)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t, bias=b, ignore_index=ignore)
    dx, dw, db = B.tbn_linear_xent_bwd(X, W, t, lse, g, bias=b, ignore_index=ignore, need_dbias=True, dw_dtype=dw_dtype)
    torch.cuda.synchronize()
    assert B.tbn_last_device_status() == (0, 0)
    for name, got in (("lse", lse), ("loss", loss), ("dx", dx), ("dw", dw), ("db", db)):
        assert_within(got, ref[name], bd[name], name)
    return loss, lse, dx, dw, db


def check_distill(x, w, bias, index, logit, tau, dloss, dw_dtype=None):
    ref = reference(x, w, bias, dloss, tau, *teacher_matrix(x.shape[0], w.shape[0], index, logit, tau))
    code = (B.F32 if x.dtype == torch.float32 else B.BF16) if dw_dtype is None else dw_dtype
    bd = bounds(ref, x, w, tau, code)
    X, W, b, i, l, g = on_gpu(x, w, bias, index, logit, dloss)
    loss, lse = B.tbn_linear_distill_fwd(X, W, i, l, temperature=tau, bias=b)
    dx, dw, db = B.tbn_linear_distill_bwd(X, W, i, l, lse, g, temperature=tau, bias=b, need_dbias=True, dw_dtype=dw_dtype)
    torch.cuda.synchronize()
    assert B.tbn_last_device_status() == (0, 0)
    for name, got in (("lse", lse), ("loss", loss), ("dx", dx), ("dw", dw), ("db", db)):
        assert_within(got, ref[name], bd[name], name)
    return loss, lse, dx, dw, db


SIZES = [(1, 8, 1), (1, 64, 200), (2, 72, 129), (64, 64, 256), (65, 128, 257), (128, 192, 1000), (257, 136, 511), (300, 320, 2050),
         (513, 64, 4097), (700, 520, 3001), (1, 500, 5000), (33, 7, 100), (130, 101, 777), (520, 1, 300), (260, 1030, 640),
         (4801, 16, 40), (2100, 64, 9001)]


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("with_bias", [False, True])
def test_cross_entropy_matches_64_bit_form(T, d, V, dtype, with_bias):
    g, x, w, bias, dloss = make(T + d + V, T, d, V, dtype, with_bias)
    targets = torch.randint(0, V, (T,), generator=g)
    targets[torch.rand(T, generator=g) < 0.2] = -100
    check_xent(x, w, bias, targets, dloss)


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K,tau", [(1, 1.0), (5, 2.0), (33, 0.5)])
def test_distillation_matches_64_bit_form(T, d, V, dtype, K, tau):
    g, x, w, bias, dloss = make(T + d + V + K, T, d, V, dtype, K == 5)
    index = torch.randint(-1, V, (T, K), generator=g)                 # repeated classes and left-out entries among them
    logit = torch.randn(T, K, generator=g) * 3
    check_distill(x, w, bias, index, logit, tau, dloss)


# ---- what a row or an entry may hold -------------------------------------------------------------------
@pytest.mark.parametrize("T", [300, 100])                        # kept rows packed to the front; rows read in place
def test_left_out_tokens_reach_nothing(T):
    """Infinities and NaN in the rows of ignored tokens, of every kind of target that is left out."""
    d, V = 64, 500
    g, x, w, bias, dloss = make(1, T, d, V, torch.bfloat16, True)
    targets = torch.randint(0, V, (T,), generator=g)
    targets[::3], targets[1::7], targets[2::11] = -100, V, -5
    left_out = (targets < 0) | (targets >= V)
    clean = check_xent(x, w, bias, targets, dloss)
    x[left_out] = torch.tensor([math.inf, -math.inf, math.nan, 3e38], dtype=torch.bfloat16).repeat(d // 4)
    dirty_dloss = dloss.clone()
    dirty_dloss[left_out] = math.nan
    dirty = check_xent(x, w, bias, targets, dirty_dloss)
    for a, b in zip(clean, dirty):
        assert torch.equal(a, b)
    assert not bool(dirty[0][left_out].any()) and not bool(dirty[1][left_out].any()) and not bool(dirty[2][left_out].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_all_tokens_left_out(dtype):
    g, x, w, bias, dloss = make(2, 70, 96, 333, dtype, True)
    out = check_xent(x, w, bias, torch.full((70,), -100), dloss)
    assert all(not bool(t.any()) for t in out)
    out = check_distill(x, w, bias, torch.full((70, 3), -1), torch.randn(70, 3, generator=g), 2.0, dloss)
    assert all(not bool(t.any()) for t in out)


def test_ignore_index_is_an_argument():
    g, x, w, bias, dloss = make(3, 40, 64, 50, torch.bfloat16, False)
    targets = torch.randint(0, 50, (40,), generator=g)
    targets[5:9] = 7
    loss, lse, dx, dw, db = check_xent(x, w, bias, targets, dloss, ignore=7)
    assert not bool(loss[5:9].any()) and bool((loss[:5][targets[:5] != 7] != 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_classes(dtype):
    """A bias of -infinity takes classes out; whole tiles of them, the first tile, and the lowest finite values."""
    T, d, V = 130, 64, 1500
    g, x, w, bias, dloss = make(4, T, d, V, dtype, True)
    bias[:600], bias[700:1030], bias[1499] = -math.inf, -math.inf, -math.inf
    bias[640:660] = torch.finfo(torch.float32).min
    allowed = torch.cat([torch.arange(600, 640), torch.arange(660, 700), torch.arange(1030, 1499)])
    targets = allowed[torch.randint(0, allowed.numel(), (T,), generator=g)]
    loss, lse, dx, dw, db = check_xent(x, w, bias, targets, dloss)
    assert bool(torch.isfinite(loss).all()) and not bool(dw[:600].any()) and not bool(db[700:1030].any())
    index = allowed[torch.randint(0, allowed.numel(), (T, 6), generator=g)]
    check_distill(x, w, bias, index, torch.randn(T, 6, generator=g), 2.0, dloss)


def test_a_target_that_is_masked_costs_infinity_and_has_a_finite_gradient():
    T, d, V = 20, 64, 300
    g, x, w, bias, dloss = make(5, T, d, V, torch.bfloat16, True)
    bias[17] = -math.inf
    targets = torch.randint(20, V, (T,), generator=g)
    targets[3] = 17
    X, W, b, t, gr = on_gpu(x, w, bias, targets, dloss)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t, bias=b)
    dx, dw, db = B.tbn_linear_xent_bwd(X, W, t, lse, gr, bias=b, need_dbias=True)
    assert math.isinf(float(loss[3])) and bool(torch.isfinite(loss[targets.to(DEV) != 17]).all())
    assert bool(torch.isfinite(lse).all()) and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
    assert abs(float(db[17]) + float(dloss[3])) < 1e-6 * float(dloss[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_bad_token_stays_alone(dtype):
    """A NaN and an infinity in kept rows reach those rows' losses and no other token's."""
    T, d, V = 200, 64, 700
    g, x, w, bias, dloss = make(6, T, d, V, dtype, False)
    x[150], x[11] = x[150].clamp(-1, 1), x[11].clamp(-1, 1)      # the largest magnitude stays in another row
    targets = torch.randint(0, V, (T,), generator=g)
    X, W, t = on_gpu(x, w, targets)
    ref, _ = B.tbn_linear_xent_fwd(X, W, t)
    X[11, 3], X[150, 0] = math.nan, math.inf
    loss, _ = B.tbn_linear_xent_fwd(X, W, t)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[11], bad[150] = True, True
    assert not bool(torch.isfinite(loss[bad]).any())
    assert torch.equal(loss[~bad], ref[~bad])


@pytest.mark.parametrize("top_dtype", [torch.float32, torch.bfloat16])
def test_teacher_entries_of_every_kind(top_dtype):
    """Left-out entries between kept ones, -infinity, the type's lowest value, a dominating entry, the same class many times."""
    T, d, V, K = 140, 64, 400, 40
    g, x, w, bias, dloss = make(7, T, d, V, torch.bfloat16, False)
    index = torch.randint(0, V, (T, K), generator=g)
    logit = (torch.randn(T, K, generator=g) * 4).to(top_dtype).float()
    index[torch.rand(T, K, generator=g) < 0.3] = -1
    index[3], logit[3] = 5, 1.0                                   # one class, forty times
    logit[4] = -math.inf                                          # nothing left
    logit[5, ::2] = -math.inf
    logit[6] = torch.finfo(top_dtype).min                         # all at the lowest finite value: uniform
    logit[7, 1:] = torch.finfo(top_dtype).min
    logit[8, 0] = 200.0
    index[9], index[10] = V, 1 << 40
    ref = reference(x, w, bias, dloss, 0.5, *teacher_matrix(T, V, index, logit, 0.5))
    bd = bounds(ref, x, w, 0.5, B.BF16)
    X, W, i, l, gr = on_gpu(x, w, index, logit.to(top_dtype), dloss)
    loss, lse = B.tbn_linear_distill_fwd(X, W, i, l, temperature=0.5)
    dx, dw, _ = B.tbn_linear_distill_bwd(X, W, i, l, lse, gr, temperature=0.5)
    for name, got in (("lse", lse), ("loss", loss), ("dx", dx), ("dw", dw)):
        assert_within(got, ref[name], bd[name], name)
    assert not bool(loss[4].any()) and not bool(dx[9:11].any())


def test_longest_list_and_a_list_as_long_as_the_vocabulary():
    g, x, w, bias, dloss = make(8, 20, 64, 3000, torch.bfloat16, False)
    index = torch.stack([torch.randperm(3000, generator=g)[:1024] for _ in range(20)])
    check_distill(x, w, bias, index, torch.randn(20, 1024, generator=g), 1.0, dloss)
    g, x, w, bias, dloss = make(9, 300, 64, 97, torch.float32, True)
    index = torch.stack([torch.randperm(97, generator=g) for _ in range(300)])
    check_distill(x, w, bias, index, torch.randn(300, 97, generator=g) * 2, 3.0, dloss)


def test_cross_entropy_is_distillation_from_one_entry():
    g, x, w, bias, dloss = make(10, 333, 128, 1111, torch.bfloat16, True)
    targets = torch.randint(0, 1111, (333,), generator=g)
    X, W, b, t, gr = on_gpu(x, w, bias, targets, dloss)
    a = B.tbn_linear_xent_fwd(X, W, t, bias=b)
    c = B.tbn_linear_distill_fwd(X, W, t[:, None].contiguous(), torch.zeros(333, 1, device=DEV), bias=b)
    assert torch.equal(a[1], c[1]) and torch.allclose(a[0], c[0], rtol=0, atol=4e-6)     # the same numbers, one more rounding of lse (|lse| < 16)
    ga = B.tbn_linear_xent_bwd(X, W, t, a[1], gr, bias=b, need_dbias=True)
    gc = B.tbn_linear_distill_bwd(X, W, t[:, None].contiguous(), torch.zeros(333, 1, device=DEV), a[1], gr, bias=b, need_dbias=True)
    for p, q in zip(ga, gc):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_several_pieces_of_the_vocabulary(dtype):
    """Enough tokens that the gradient is taken in several pieces; dX is summed over them."""
    T, d, V = 40000 if dtype == torch.bfloat16 else 20000, 24, 9000
    g, x, w, bias, dloss = make(11, T, d, V, dtype, True)
    targets = torch.randint(0, V, (T,), generator=g)
    targets[torch.rand(T, generator=g) < 0.5] = -100
    check_xent(x, w, bias, targets, dloss, dw_dtype=B.F32)
    index = torch.randint(0, V, (T, 2), generator=g)
    X, W, b, i, l, gr = on_gpu(x, w, bias, index, torch.randn(T, 2, generator=g), dloss)
    loss, lse = B.tbn_linear_distill_fwd(X, W, i, l, bias=b)
    assert bool(torch.isfinite(loss).all())


@pytest.mark.parametrize("dtype,dw_dtype", [(torch.bfloat16, B.F32), (torch.float32, B.BF16), (torch.bfloat16, B.BF16)])
def test_type_of_dw(dtype, dw_dtype):
    g, x, w, bias, dloss = make(12, 200, 72, 600, dtype, False)
    out = check_xent(x, w, bias, torch.randint(0, 600, (200,), generator=g), dloss, dw_dtype=dw_dtype)
    assert out[3].dtype == (torch.float32 if dw_dtype == B.F32 else torch.bfloat16) and out[2].dtype == dtype


def test_signed_and_zero_loss_gradients():
    g, x, w, bias, dloss = make(13, 150, 64, 320, torch.float32, True)
    dloss[::2] *= -3.0
    dloss[1::5] = 0.0
    check_xent(x, w, bias, torch.randint(0, 320, (150,), generator=g), dloss)
    check_xent(x, w, bias, torch.randint(0, 320, (150,), generator=g), torch.zeros(150))


@pytest.mark.parametrize("T", [171, 300])
def test_a_mean_of_any_number_of_tokens_is_not_off_as_a_whole(T):
    """256 classes of one logit each: every q is 2^-8, so every dz / dloss is 2^-8 or 2^-8 - 1, which bf16 holds exactly.  With
    one dloss for all tokens that leaves the sums' own error: (T / 16 + 8) cut-offs of 2^-23 (the 8 cover the factor taken out
    and put back and the output's rounding to fp32).  1 / T itself is 0.2 % off in bf16 for both T."""
    d, V = 64, 256
    g, x, w, _, _ = make(T, T, d, V, torch.bfloat16, False)
    x[:, -1] = 0
    w[:, :-1] = 0
    dloss = torch.full((T,), 1.0 / T)
    targets = torch.randint(0, V, (T,), generator=g)
    targets[::5] = -100
    _, _, dx, dw, db = check_xent(x, w, None, targets, dloss, dw_dtype=B.F32)
    ref = reference(x, w, None, dloss, 1.0, *one_hot(targets, V))
    assert_within(dw, ref["dw"], ref["dw_abs"] * (T / 16 + 8) * 2.0 ** -23, "dw")
    assert_within(dx, ref["dx"], ref["dx_abs"] * (V / 16 + 8) * 2.0 ** -23 + ref["dx"].abs() * 2.0 ** -8, "dx")


@pytest.mark.parametrize("scale_x,scale_w", [(1e-12, 1e10), (1e8, 1e-9), (1e-3, 1e-3)])
def test_fp32_operands_of_any_magnitude(scale_x, scale_w):
    g, x, w, bias, dloss = make(14, 90, 80, 300, torch.float32, False)
    check_xent(x * scale_x, w * scale_w, bias, torch.randint(0, 300, (90,), generator=g), dloss * 1e-6)


# ---- parts of the gradient, buffers, streams, graphs --------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_subset_of_the_gradients(dtype):
    g, x, w, bias, dloss = make(20, 270, 88, 900, dtype, True)
    X, W, b, t, gr = on_gpu(x, w, bias, torch.randint(-1, 900, (270,), generator=g), dloss)
    _, lse = B.tbn_linear_xent_fwd(X, W, t, bias=b)
    full = B.tbn_linear_xent_bwd(X, W, t, lse, gr, bias=b, need_dbias=True)
    for want in range(8):
        got = B.tbn_linear_xent_bwd(X, W, t, lse, gr, bias=b, need_dx=bool(want & 1), need_dw=bool(want & 2), need_dbias=bool(want & 4))
        for k in range(3):
            assert (got[k] is None) == (not want >> k & 1)
            # splits of a contraction follow from the sizes, not from what is asked for: the same bits
            assert got[k] is None or torch.equal(got[k], full[k]), (want, k)


def guarded(shape, dtype):
    n = math.prod(shape)
    size = torch.empty((), dtype=dtype).element_size()
    buf = torch.full((16384 + n * size + (-n * size) % 256,), 0xA5, dtype=torch.uint8, device=DEV)
    return buf, buf[8192:8192 + n * size].view(dtype).view(*shape)


@pytest.mark.parametrize("T,d,V", [(1, 72, 129), (130, 104, 1001), (257, 33, 515), (300, 16, 70), (64, 500, 260)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_and_workspace_stay_inside_their_buffers(T, d, V, dtype):
    g, x, w, bias, dloss = make(21, T, d, V, dtype, True)
    X, W, b, t, gr = on_gpu(x, w, bias, torch.randint(-1, V, (T,), generator=g), dloss)
    code = B.BF16 if dtype == torch.bfloat16 else B.F32
    for back in (False, True):
        need = B.tbn_linear_xent_workspace_bytes(T, d, V, code, back)
        bufs = [guarded((need,), torch.uint8)]
        ws = bufs[0][1]
        lib, p = B.lib(), lambda q: q.data_ptr()
        if not back:
            bufs += [guarded((T,), torch.float32), guarded((T,), torch.float32)]
            assert lib.tbn_linear_xent_fwd(p(X), p(W), code, T, d, V, p(b), p(t), -100, p(bufs[1][1]), p(bufs[2][1]), p(ws), need, B._stream()) == 0
            lse = bufs[2][1].clone()
        else:
            bufs += [guarded((T, d), dtype), guarded((V, d), torch.float32), guarded((V,), torch.float32)]
            assert lib.tbn_linear_xent_bwd(p(X), p(W), code, T, d, V, p(b), p(t), -100, p(lse), p(gr), p(bufs[1][1]), p(bufs[2][1]), B.F32,
                                           p(bufs[3][1]), p(ws), need, B._stream()) == 0
        torch.cuda.synchronize()
        for buf, out in bufs:
            n = out.numel() * out.element_size()
            assert bool((buf[:8192] == 0xA5).all()) and bool((buf[8192 + n:] == 0xA5).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_results_do_not_depend_on_what_the_workspace_held(dtype):
    T, d, V, K = 290, 200, 1300, 9
    g, x, w, bias, dloss = make(22, T, d, V, dtype, True)
    index, logit = torch.randint(-1, V, (T, K), generator=g), torch.randn(T, K, generator=g)
    index[::4] = -1
    X, W, b, i, l, gr = on_gpu(x, w, bias, index, logit, dloss)
    code = B.BF16 if dtype == torch.bfloat16 else B.F32
    runs = []
    for fill in (0, 0xFF, 0x7F):
        ws = [torch.full((B.tbn_linear_distill_workspace_bytes(T, d, V, code, K, back),), fill, dtype=torch.uint8, device=DEV) for back in (0, 1)]
        loss, lse = B.tbn_linear_distill_fwd(X, W, i, l, 1.5, bias=b, workspace=ws[0])
        runs.append((loss, lse) + B.tbn_linear_distill_bwd(X, W, i, l, lse, gr, 1.5, bias=b, need_dbias=True, workspace=ws[1]))
    for r in runs[1:]:
        for p, q in zip(runs[0], r):
            assert torch.equal(p, q)


def test_a_stream_of_its_own_and_two_calls_at_once():
    T, d, V = 600, 256, 5000
    cases = []
    for seed in (23, 24):
        g, x, w, bias, dloss = make(seed, T, d, V, torch.bfloat16, False)
        X, W, t, gr = on_gpu(x, w, torch.randint(0, V, (T,), generator=g), dloss)
        loss, lse = B.tbn_linear_xent_fwd(X, W, t)
        cases.append((X, W, t, gr, (loss, lse) + B.tbn_linear_xent_bwd(X, W, t, lse, gr)[:2]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for k, (X, W, t, gr, _) in enumerate(cases):
            with torch.cuda.stream(streams[k]):
                loss, lse = B.tbn_linear_xent_fwd(X, W, t)
                got[k].append((loss, lse) + B.tbn_linear_xent_bwd(X, W, t, lse, gr)[:2])
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            for p, q in zip(cases[k][4], r):
                assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_step_replayed_on_new_inputs(dtype):
    T, d, V, K = 180, 96, 700, 4
    g, x, w, bias, dloss = make(25, T, d, V, dtype, True)
    index, logit = torch.randint(-1, V, (T, K), generator=g), torch.randn(T, K, generator=g)
    X, W, b, i, l, gr = on_gpu(x, w, bias, index, logit, dloss)
    t = i[:, 0].contiguous()

    def step():
        loss, lse = B.tbn_linear_xent_fwd(X, W, t, bias=b)
        out = (loss, lse) + B.tbn_linear_xent_bwd(X, W, t, lse, gr, bias=b, need_dbias=True)
        loss, lse = B.tbn_linear_distill_fwd(X, W, i, l, 2.0, bias=b)
        return out + (loss, lse) + B.tbn_linear_distill_bwd(X, W, i, l, lse, gr, 2.0, bias=b, need_dbias=True)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (26, 27):
        g2, x2, w2, bias2, dloss2 = make(seed, T, d, V, dtype, True)
        for dst, src in ((X, x2), (W, w2), (b, bias2), (gr, dloss2)):
            dst.copy_(src)
        i.copy_(torch.randint(-1, V, (T, K), generator=g2))
        t.copy_(i[:, 0])
        if seed == 27:
            t.fill_(-100)                      # another number of kept tokens than at capture
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        for p, q in zip(got, step()):
            assert torch.equal(p, q)


def test_tiled_head_trained_through_the_loss():
    """The calls as a training step strings them: B_hat from W, loss and G from the head, dW from G; against the same chain
    in 64 bits.  B_hat is given (its bits are tested elsewhere), so the errors are those of G: bounds() and one more sum."""
    T, d, V, k = 260, 128, 512, 4
    g = torch.Generator().manual_seed(30)
    Wf = torch.randn(V, d, generator=g) * 0.1
    x = torch.randn(T, d, generator=g).to(torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=g)
    dloss = torch.full((T,), 1.0 / T)
    Wd, X, t, gr = on_gpu(Wf, x, targets, dloss)
    B_hat, tile, alpha = B.tbn_tile_fwd(Wd, k, B.ALPHA_PER_TILE, b_dtype=B.BF16)
    head = B_hat.view(V, d)
    loss, lse = B.tbn_linear_xent_fwd(X, head, t)
    dx, G, _ = B.tbn_linear_xent_bwd(X, head, t, lse, gr, dw_dtype=B.F32)
    dW, _, dalpha = B.tbn_tile_bwd(G.view(-1), tile, alpha, Wd.view(-1), k, B.ALPHA_PER_TILE)
    torch.cuda.synchronize()
    ref = reference(x, head, None, dloss, 1.0, *one_hot(targets, V))
    bd = bounds(ref, x, head, 1.0, B.F32)
    for name, got in (("loss", loss), ("dx", dx), ("dw", G)):
        assert_within(got, ref[name], bd[name], name)
    q = V * d // k
    S, a = Wd.double().view(k, q), alpha.double()[:, None]
    t_signs = torch.where(S.sum(0) > 0, 1.0, -1.0).double()
    Gr, Gb = ref["dw"].view(k, q), bd["dw"].view(k, q)
    dal = (Gr * t_signs).sum(1)
    dal_b = Gb.sum(1) + 1e-6 * Gr.abs().sum(1)
    assert_within(dalpha, dal, dal_b, "dalpha")
    want = a * Gr + dal[:, None] * S.sign() / q
    assert_within(dW.view(k, q), want, a * Gb + dal_b[:, None] / q + 1e-6 * (a * Gr).abs() + 1e-6 * dal.abs()[:, None] / q, "dW")


def test_gradient_against_differences_of_the_loss():
    """The kernels' own loss at shifted weights: fp32, a shift large enough that the loss moves by many of its roundings."""
    T, d, V = 64, 40, 90
    g, x, w, bias, dloss = make(31, T, d, V, torch.float32, True)
    targets = torch.randint(0, V, (T,), generator=g)
    X, W, b, t, gr = on_gpu(x, w, bias, targets, dloss)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t, bias=b)
    dx, dw, db = B.tbn_linear_xent_bwd(X, W, t, lse, gr, bias=b, need_dbias=True)
    u = torch.randn(V, d, generator=g).to(DEV)
    u /= u.norm()
    h = 0.05
    total = lambda Wt: float((B.tbn_linear_xent_fwd(X, Wt, t, bias=b)[0].double() * gr.double()).sum())
    slope = (total(W + h * u) - total(W - h * u)) / (2 * h)
    want = float((dw.double() * u.double()).sum())
    # the central difference is off by h^2 / 6 times a third derivative along u (the logits move by |x . u_v| <= |x||u_v|, the
    # third derivative of a softmax loss is below 8 of their cube), and by the roundings of the two losses over 2 h
    move = (X.double().norm(dim=1)[:, None] * u.double().norm(dim=1)[None, :]).max(1).values
    third = float((gr.double() * 8 * move ** 3).sum())
    rounding = float(gr.sum()) * 2.0 ** -19 * 8 / h
    assert abs(slope - want) <= h * h / 6 * third + rounding


# ---- lengths ---------------------------------------------------------------------------------------------------
def test_no_tokens():
    X, W = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV), torch.ones(30, 64, dtype=torch.bfloat16, device=DEV)
    t, f = torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, device=DEV)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t)
    assert loss.shape == lse.shape == (0,)
    dx, dw, db = B.tbn_linear_xent_bwd(X, W, t, lse, f, need_dbias=True)
    assert dx.shape == (0, 64) and not bool(dw.any()) and not bool(db.any())
    loss, lse = B.tbn_linear_distill_fwd(X, W, t.view(0, 1).expand(0, 3).contiguous(), f.view(0, 1).expand(0, 3).contiguous())
    assert loss.shape == (0,)


def test_offsets_beyond_32_bits_in_the_activations():
    """x and dx of more than 2^32 bytes; the tokens at both ends and in the middle against the 64-bit form."""
    T, d, V = 1_100_000, 2048, 9
    X = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(40)
    rows = torch.tensor([0, 1, 255, 256, T // 2, 1_048_575, 1_048_576, 1_048_577, T - 2, T - 1], device=DEV)
    X[rows] = torch.randn(rows.numel(), d, generator=g, device=DEV).to(torch.bfloat16)
    W = (torch.randn(V, d, generator=g, device=DEV) / math.sqrt(d)).to(torch.bfloat16)
    t = torch.full((T,), -100, dtype=torch.int64, device=DEV)
    t[rows] = torch.arange(rows.numel(), device=DEV) % V
    t[::100_003] = 2
    kept = (t >= 0).nonzero()[:, 0]
    gr = torch.ones(T, device=DEV)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t)
    dx, dw, _ = B.tbn_linear_xent_bwd(X, W, t, lse, gr)
    x, targets = X[kept].cpu(), t[kept].cpu()
    ref = reference(x, W.cpu(), None, torch.ones(kept.numel()), 1.0, *one_hot(targets, V))
    bd = bounds(ref, x, W, 1.0, B.BF16)
    for name, got in (("loss", loss[kept]), ("lse", lse[kept]), ("dx", dx[kept]), ("dw", dw)):
        assert_within(got, ref[name], bd[name], name)
    assert int((loss != 0).sum()) <= kept.numel() and int((dx.view(torch.int16)[:, 0] != 0).sum()) <= kept.numel()
    # and with every token kept, so that the packed rows and the pieces of dz are that large as well
    t[:] = torch.arange(T, device=DEV) % V
    loss, lse = B.tbn_linear_xent_fwd(X, W, t)
    gr = torch.full((T,), 1.0 / T, device=DEV)
    dx, dw, db = B.tbn_linear_xent_bwd(X, W, t, lse, gr, need_dbias=True)
    z = X[rows].double() @ W.double().t()
    assert float((lse[rows].double() - torch.logsumexp(z, 1)).abs().max()) < 1e-4
    q = torch.softmax(z, 1)
    q[torch.arange(rows.numel(), device=DEV), t[rows]] -= 1
    want = (q / T) @ W.double()
    assert float((dx[rows].double() - want).abs().max()) <= 2.0 ** -7 * float(((q.abs() / T) @ W.double().abs()).max())
    assert abs(float(db.double().sum())) < 1e-5


def test_offsets_beyond_32_bits_in_the_weights():
    T, d, V = 3, 2048, 1_100_000
    g = torch.Generator(device=DEV).manual_seed(41)
    X = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    W = torch.randn(V, d, generator=g, device=DEV, dtype=torch.bfloat16) * 0.02
    t = torch.tensor([V - 1, 0, 1_048_577], device=DEV)
    gr = torch.ones(T, device=DEV)
    loss, lse = B.tbn_linear_xent_fwd(X, W, t)
    dx, dw, _ = B.tbn_linear_xent_bwd(X, W, t, lse, gr)
    z = torch.cat([X.double() @ W[a:a + 100_000].double().t() for a in range(0, V, 100_000)], 1)
    ref = torch.logsumexp(z, 1)
    # z: d / 16 + 8 steps of 2^-23 of a sum of |x||w| below 2048 * 0.02 * 0.7 = 30
    assert float((lse.double() - ref).abs().max()) < 2 * 30 * (2048 / 16 + 8) * 2.0 ** -23 + 2.0 ** -18
    assert float((loss.double() - (ref - z[torch.arange(T, device=DEV), t])).abs().max()) < 4 * 30 * (2048 / 16 + 8) * 2.0 ** -23 + 2.0 ** -17
    q = torch.softmax(z, 1)
    q[torch.arange(T, device=DEV), t] -= 1
    for a in (0, 1_048_500, V - 100):
        want = q[:, a:a + 100].t() @ X.double()
        size = q[:, a:a + 100].abs().t() @ X.double().abs()
        assert bool(((dw[a:a + 100].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1e-4) * size).all())
