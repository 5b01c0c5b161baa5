"""LayerNorm's gradient of rows that lie far from zero in units of their deviation, so far that mean * rstd is beyond the largest float:
every x - mean is 0, all of the inputs are finite, and so is every gradient."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
FAR, RSTD = 2.0 ** 110, 2.0 ** 20                                       # as eps = 2^-40 gives it for a row without deviation


def check(T, d, dtype, rows, affine, dsum):
    """The rows `rows` far, the others ordinary ones."""
    g = torch.Generator(device=DEV).manual_seed(T + d)
    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    s, dy = randn(T, d).to(dtype), randn(T, d).to(dtype)
    mean, rstd = s.float().mean(1), torch.ones(T, device=DEV)
    s[rows], mean[rows], rstd[rows] = FAR, FAR, RSTD
    gamma = 1 + 0.2 * randn(d) if affine else None
    other = randn(T, d).to(dtype) if dsum else None
    dx, dgamma, dbeta = B.tbn_layernorm_bwd(dy, s, mean, rstd, gamma, dsum=other)
    r = rstd.double()[:, None]
    h, a = (s.double() - mean.double()[:, None]) * r, dy.double() * (gamma.double() if affine else 1.0)
    m1, m2 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    want = r * (a - m1 - h * m2) + (other.double() if dsum else 0.0)
    # roundings of u: a row's sums in at most 48 + d / 256 steps, eight more of their terms and of what is put together
    n = 56 + d // 256
    err = r * U * (8 * a.abs() + 8 * (h * m2).abs() + n * (a.abs().mean(1, keepdim=True) + h.abs() * (a * h).abs().mean(1, keepdim=True)))
    err += (2 * U + torch.finfo(dtype).eps / 2 * 1.01) * want.abs() + 1e-40
    assert torch.isfinite(dx).all() and torch.isfinite(dgamma).all() and torch.isfinite(dbeta).all()
    assert ((dx.double() - want).abs() <= err).all()
    depth = 68 + T // 64                                                # roundings in a row of a column's sum
    gd = dy.double()
    assert ((dgamma.double() - (gd * h).sum(0)).abs() <= depth * U * (gd * h).abs().sum(0)).all()
    assert ((dbeta.double() - gd.sum(0)).abs() <= depth * U * gd.abs().sum(0)).all()


# every way in which a row leaves lanes or parts of a piece without columns: empty lanes of a row's 4 to 32, of its last warp, ends of
# rows that are not whole pieces, the second row of them beginning inside a piece; long rows last
@pytest.mark.parametrize("d", [1, 24, 25, 40, 63, 96, 100, 255, 300, 501, 1000, 1500, 2040, 2047, 4098, 8185, 9001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("affine,dsum", [(False, False), (True, True)])
def test_columns_that_a_row_does_not_have(d, dtype, affine, dsum):
    check(8, d, dtype, slice(None), affine, dsum)
    check(8, d, dtype, slice(3, 5), affine, dsum)
