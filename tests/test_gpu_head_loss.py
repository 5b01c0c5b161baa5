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
