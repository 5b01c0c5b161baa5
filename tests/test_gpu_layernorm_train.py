"""LayerNorm for training against the formulas in 64 bits.

u = 2^-24.  A row's sums have at most `chain` roundings one after another (32 values of a thread, or d / 256 of them in long
rows, five and up to eight joins), so a sum's error is at most chain u times the sum of magnitudes."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def chain(d):
    return 48 + d // 256


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rand(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    over = (err - bound).max().item() if err.numel() else 0.0
    assert not math.isnan(over) and over <= 0, f"{what}: {err.max().item()} off, {over} over its bound"


def case(T, d, x_dtype, y_dtype, residual, affine, seed=0):
    x = rand(seed, T, d, dtype=DT[x_dtype], scale=1.5) + 0.5
    r = rand(seed + 1, T, d, dtype=DT[x_dtype]) if residual else None
    gamma = 1 + rand(seed + 2, d, scale=0.2) if affine else None
    beta = rand(seed + 3, d, scale=0.2) if affine else None
    dy = rand(seed + 4, T, d, dtype=DT[y_dtype])
    dsum = rand(seed + 5, T, d, dtype=DT[x_dtype]) if residual else None
    return x.to(DT[x_dtype]), r, gamma, beta, dy, dsum


SHAPES = [(1, 1), (3, 2), (2, 31), (5, 64), (1, 255), (7, 256), (9, 257), (33, 501), (4, 768), (1000, 96), (130, 1024), (17, 2047), (6, 2048), (5, 2056),
          (3, 4096), (2, 4097), (3, 8192), (2, 8200), (2, 20001), (3000, 40), (1, 8200), (1, 8192), (1, 20001), (32, 512), (33, 512), (16, 255), (70, 20001), (500, 32), (77, 16), (5000, 24), (301, 63), (900, 100), (129, 128), (1300, 121)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("residual,affine", [(False, True), (True, True), (True, False)])
def test_forward_and_backward(T, d, x_dtype, y_dtype, residual, affine):
    eps = 1e-5
    x, r, gamma, beta, dy, dsum = case(T, d, x_dtype, y_dtype, residual, affine)
    y, s, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, eps, residual=r, y_dtype=B.F32 if y_dtype == "f32" else B.BF16)
    want_s = x if r is None else (x.float() + r.float()).to(x.dtype)
    assert torch.equal(s, want_s)
    z = want_s.double()
    w, o = (gamma.double(), beta.double()) if affine else (1.0, 0.0)
    n = chain(d)
    var, mu = torch.var_mean(z, 1, correction=0, keepdim=True)
    rs = (var + eps).rsqrt()
    size = z.abs().mean(1, keepdim=True)
    mean_err = n * U * size + U * mu.abs()
    within(mean[:, None], mu, mean_err, "mean")
    # the variance: its own roundings (of a sum of squares, each of a difference that is u off), and the square of the mean's error
    rstd_err = rs * (0.5 * rs ** 2 * ((n + 8) * U * var + mean_err ** 2 + 2 * mean_err * U * z.abs().amax(1, keepdim=True)) + 4 * U)
    within(rstd[:, None], rs, rstd_err, "rstd")
    h = (z - mu) * rs
    err = (h.abs() * (rstd_err / rs + 4 * U) + (mean_err + U * z.abs()) * rs) * (w if affine else 1.0)
    want = h * w + o
    within(y, want, err.abs() + 2 * U * want.abs() + 2 * U * (h * w).abs() + half_step(y.dtype) * want.abs() * 1.01 + 1e-40, "y")

    # the backward from the statistics as they are in 32 bits, so that only its own roundings count
    dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma, dsum=dsum)
    h = (z - mean.double()[:, None]) * rstd.double()[:, None]
    a = dy.double() * w
    m1, m2 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    want = rstd.double()[:, None] * (a - m1 - h * m2)
    err = rstd.double()[:, None] * U * (8 * a.abs() + 8 * m1.abs() + 8 * (h * m2).abs() + (n + 8) * (a.abs().mean(1, keepdim=True) + h.abs() * (a * h).abs().mean(1, keepdim=True)))
    if dsum is not None:
        want = want + dsum.double()
    within(dx, want, err + (2 * U + half_step(dx.dtype) * 1.01) * want.abs() + 1e-40, "dx")
    assert dx.dtype == x.dtype
    depth = 64 + T // 64                                                # roundings in a row of a column's sum: rows of a block, blocks
    g = dy.double()
    within(dgamma, (g * h).sum(0), (depth + 4) * U * (g * h).abs().sum(0), "dgamma")
    within(dbeta, g.sum(0), depth * U * g.abs().sum(0), "dbeta")


def test_gradient_against_differences():
    """sum(y * g) as a function of x, gamma and beta, in 64 bits from the definition."""
    T, d = 5, 37
    x, _, gamma, beta, dy, _ = case(T, d, "f32", "f32", False, True, seed=40)
    _, s, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, 1e-5)
    dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma)

    def f(x, gamma, beta):
        var, mu = torch.var_mean(x, 1, correction=0, keepdim=True)
        return (((x - mu) / torch.sqrt(var + 1e-5) * gamma + beta) * dy.double()).sum()
    args = [x.double(), gamma.double(), beta.double()]
    step = 1e-5
    for i, got in enumerate((dx, dgamma, dbeta)):
        for at in range(0, got.numel(), 7):
            moved = [[a.clone() for a in args] for _ in range(2)]
            moved[0][i].view(-1)[at] += step
            moved[1][i].view(-1)[at] -= step
            want = (f(*moved[0]) - f(*moved[1])).item() / (2 * step)
            # differences: step^2 / 6 of a third derivative of a few units (1e-9), 64-bit noise 1e-10; the kernel: 200 u of sums below 100
            assert abs(got.view(-1)[at].item() - want) < 2e-5 + 1e-6 * abs(want)


def test_constant_rows_and_bad_rows_stay_to_themselves():
    T, d = 40, 300
    x, _, gamma, beta, dy, _ = case(T, d, "f32", "f32", False, True, seed=50)
    x[3] = 7.0                                                          # no variance: h = 0
    x[5, 17], x[9, 0] = float("inf"), float("nan")
    y, s, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, 1e-5)
    assert torch.equal(y[3], beta)
    ok = [t for t in range(T) if t not in (5, 9)]
    assert torch.isfinite(y[ok]).all() and torch.isnan(y[[5, 9]]).all()
    dx, dgamma, _ = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma)
    assert torch.isfinite(dx[ok]).all() and torch.isnan(dx[[5, 9]]).all() and torch.isnan(dgamma).all()


def test_large_offset_keeps_its_variance():
    """Rows of 1000 + noise of 1: the second moment is taken around the mean.  The mean is off by up to 64 u 1000 = 4e-3, which enters
    the variance squared, and each x - mean by 6e-5."""
    x = rand(60, 64, 1500) + 1000.0
    _, _, mean, rstd = B.tbn_layernorm_train_fwd(x)
    var = x.double().var(1, correction=0)
    assert ((rstd.double() - (var + 1e-5).rsqrt()).abs() < 1e-4).all()


def test_empty_batches_and_outputs_left_out():
    gamma = torch.ones(64, device=DEV)
    y, s, mean, rstd = B.tbn_layernorm_train_fwd(torch.empty(0, 64, device=DEV), gamma)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dgamma, dbeta = B.tbn_layernorm_bwd(y, s, mean, rstd, gamma)
    assert dx.shape == (0, 64) and not dgamma.any() and not dbeta.any()
    x, _, gamma, _, dy, _ = case(20, 64, "bf16", "bf16", False, True)
    _, s, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma)
    full = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma)
    for need in ((True, False), (False, True), (False, False)):
        got = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma, need_dgamma=need[0], need_dbeta=need[1])
        assert torch.equal(got[0], full[0])
        for k in (0, 1):
            assert torch.equal(got[1 + k], full[1 + k]) if need[k] else got[1 + k] is None


def test_rows_of_three_dimensions_give_the_same():
    x, r, gamma, beta, dy, dsum = case(24, 96, "bf16", "bf16", True, True)
    shaped = lambda t: t.view(2, 12, 96)  # noqa: E731
    a = B.tbn_layernorm_train_fwd(x, gamma, beta, residual=r)
    b = B.tbn_layernorm_train_fwd(shaped(x), gamma, beta, residual=shaped(r))
    assert torch.equal(a[0], b[0].view(24, 96)) and b[0].shape == (2, 12, 96)
    c = B.tbn_layernorm_bwd(dy, *a[1:], gamma, dsum=dsum)
    e = B.tbn_layernorm_bwd(shaped(dy), *b[1:], gamma, dsum=shaped(dsum))
    assert all(torch.equal(p.reshape(-1), q.reshape(-1)) for p, q in zip(c, e))


@pytest.mark.parametrize("d", [501, 768, 9000])
def test_nothing_is_written_outside_the_outputs_and_bits_repeat(d):
    """Outputs inside larger buffers, through the C entry points; a workspace full of NaN changes nothing."""
    T, pad = 37, 64
    x, r, gamma, beta, dy, dsum = case(T, d, "bf16", "bf16", True, True, seed=70)
    need = B.tbn_layernorm_bwd_workspace_bytes(T, d)
    runs = []
    for fill in (float("nan"), 3.0):
        room = lambda n, dt: torch.full((n + 2 * pad,), 5.0, dtype=dt, device=DEV)  # noqa: E731
        s, y, dx = (room(T * d, torch.bfloat16) for _ in range(3))
        mean, rstd, dg, db = room(T, torch.float32), room(T, torch.float32), room(d, torch.float32), room(d, torch.float32)
        ws = torch.full((need // 4 + 1 + 2 * pad,), fill, dtype=torch.float32, device=DEV)
        at = lambda t: t.data_ptr() + pad * t.element_size()  # noqa: E731
        stream = torch.cuda.current_stream().cuda_stream
        assert B.lib().tbn_layernorm_train_fwd(x.data_ptr(), r.data_ptr(), B.BF16, T, d, gamma.data_ptr(), beta.data_ptr(), 1e-5, at(s), at(y), B.BF16,
                                               at(mean), at(rstd), stream) == 0
        assert B.lib().tbn_layernorm_bwd(dy.data_ptr(), B.BF16, at(s), B.BF16, T, d, gamma.data_ptr(), at(mean), at(rstd), dsum.data_ptr(), at(dx), at(dg),
                                         at(db), at(ws), need, stream) == 0
        torch.cuda.synchronize()
        outs = [s, y, dx, mean, rstd, dg, db]
        for t in outs:
            assert (t[:pad] == 5).all() and (t[-pad:] == 5).all()
            assert not torch.isnan(t).any()
        edge = torch.cat([ws[:pad], ws[need // 4 + pad:]])
        assert (torch.isnan(edge) if math.isnan(fill) else edge == fill).all()
        runs.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("d", [96, 501, 1500, 2050])
def test_a_row_does_not_depend_on_the_batch(d):
    """y, dx and the statistics of a row are the same bits alone, among a few rows and among many.  Rows that are not whole pieces of eight
    columns are added up from the aligned piece on that they begin in, in another order where they begin elsewhere: there the row's place
    in its piece has to be the same."""
    T, same = 1200, 8 // math.gcd(d, 8)
    x, r, gamma, beta, dy, dsum = case(T, d, "bf16", "bf16", True, True, seed=80)
    many = B.tbn_layernorm_train_fwd(x, gamma, beta, residual=r)
    dx = B.tbn_layernorm_bwd(dy, *many[1:], gamma, dsum=dsum)[0]
    for a, b in ((0, 1), (5, 8), (1100, 1160)):
        a = a // same * same
        few = B.tbn_layernorm_train_fwd(x[a:b].clone(), gamma, beta, residual=r[a:b].clone())
        assert all(torch.equal(p, q[a:b]) for p, q in zip(few, many))
        assert torch.equal(B.tbn_layernorm_bwd(dy[a:b].clone(), *few[1:], gamma, dsum=dsum[a:b].clone())[0], dx[a:b])


def test_two_streams_at_once():
    jobs = [case(3000, d, "bf16", "bf16", True, True, seed=90 + d) for d in (768, 501)]

    def run(job):
        x, r, gamma, beta, dy, dsum = job
        y, *kept = B.tbn_layernorm_train_fwd(x, gamma, beta, residual=r)
        return (y, *kept, *B.tbn_layernorm_bwd(dy, *kept, gamma, dsum=dsum))
    want = [run(j) for j in jobs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in jobs], []
    for _ in range(4):
        for j, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                got.append(run(j))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
