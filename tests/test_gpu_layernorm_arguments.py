"""LayerNorm for training: what may be left out or be given without need, rows beside rows with an infinity or a NaN, the widest rows."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.test_gpu_layernorm_train import DEV, DT, U, case, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [40, 63, 1024, 8200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_statistics_left_out_and_a_sum_without_need(d, dtype):
    T = 21
    x, r, gamma, beta, _, _ = case(T, d, dtype, dtype, True, True, seed=300)
    code = B.F32 if dtype == "f32" else B.BF16
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    for residual in (None, r):
        for g, b in ((gamma, None), (None, beta), (None, None)):
            want, s, mean, rstd = B.tbn_layernorm_train_fwd(x, g, b, residual=residual)
            for m, v in ((None, None), (torch.zeros_like(mean), None), (None, torch.zeros_like(rstd))):
                y, total = torch.zeros_like(x), torch.full_like(x, 5.0)
                assert B.lib().tbn_layernorm_train_fwd(ptr(x), ptr(residual), code, T, d, ptr(g), ptr(b), 1e-5, ptr(total), ptr(y), code, ptr(m), ptr(v),
                                                       torch.cuda.current_stream().cuda_stream) == 0
                assert torch.equal(y, want)
                assert (total == 5.0).all() if residual is None else torch.equal(total, s)
                assert m is None or torch.equal(m, mean)
                assert v is None or torch.equal(v, rstd)


@pytest.mark.parametrize("d", [1, 7, 24, 25, 63, 100, 128, 255, 501, 1500, 2047, 4098, 8187, 9001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_beside_bad_ones_keep_their_bits(d, dtype):
    """Rows of odd widths share 16 bytes with their neighbours, narrow ones a warp."""
    T = 100
    x, r, gamma, beta, dy, dsum = case(T, d, dtype, dtype, True, True, seed=310)
    clean = B.tbn_layernorm_train_fwd(x, gamma, beta, residual=r)
    grad = B.tbn_layernorm_bwd(dy, *clean[1:], gamma, dsum=dsum)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[[0, 7, 8, 50, 99]] = True
    for value in (float("nan"), float("inf")):
        x2, dy2 = x.clone(), dy.clone()
        x2[bad] = value
        got = B.tbn_layernorm_train_fwd(x2, gamma, beta, residual=r)
        assert all(torch.equal(a[~bad], b[~bad]) for a, b in zip(got, clean))
        assert torch.isnan(got[0][bad]).all()
        dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy, *got[1:], gamma, dsum=dsum)
        assert torch.equal(dx[~bad], grad[0][~bad]) and torch.isnan(dx[bad]).all() and torch.isnan(dgamma).all() and torch.equal(dbeta, grad[2])
        dy2[bad] = value
        dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy2, *clean[1:], gamma, dsum=dsum)
        assert torch.equal(dx[~bad], grad[0][~bad]) and torch.isnan(dx[bad]).all() and not torch.isfinite(dgamma).any() and not torch.isfinite(dbeta).any()


def test_the_widest_rows():
    """2^23 columns: a thread adds 32768 of them one after another, and partial sums of a column's rows are few."""
    T, d = 3, 2 ** 23
    x, r, gamma, beta, dy, dsum = case(T, d, "bf16", "bf16", True, True, seed=320)
    y, s, mean, rstd = B.tbn_layernorm_train_fwd(x, gamma, beta, residual=r)
    z = s.double()
    var, mu = torch.var_mean(z, 1, correction=0, keepdim=True)
    n = 32768 + 16
    within(mean[:, None], mu, n * U * z.abs().mean(1, keepdim=True), "mean")
    rs = (var + 1e-5).rsqrt()
    within(rstd[:, None], rs, rs * (n + 8) * U + rs * 4 * U, "rstd")
    m64, r64 = mean.double()[:, None], rstd.double()[:, None]
    h, half = (z - m64) * r64, torch.finfo(torch.bfloat16).eps / 2 * 1.01
    want = h * gamma.double() + beta.double()
    within(y, want, 6 * U * ((z.abs() + m64.abs()) * r64 * gamma.double().abs() + want.abs()) + half * want.abs(), "y")
    dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma, dsum=dsum)
    a = dy.double() * gamma.double()
    m1, m2 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    want = r64 * (a - m1 - h * m2) + dsum.double()
    err = r64 * U * (8 * a.abs() + 8 * (h * m2).abs() + n * (a.abs().mean(1, keepdim=True) + h.abs() * (a * h).abs().mean(1, keepdim=True)))
    within(dx, want, err + (2 * U + half) * want.abs(), "dx")
    within(dgamma, (dy.double() * h).sum(0), 12 * U * (dy.double() * h).abs().sum(0), "dgamma")
    within(dbeta, dy.double().sum(0), 8 * U * dy.double().abs().sum(0), "dbeta")
