"""Head losses without a GPU: refusals answered on the host before anything is launched, workspace queries, and the plain
64-bit form the GPU tests compare with, held against finite differences."""
import math

import pytest
import torch

from paper_2407_12075_b200 import binding as B
from paper_2407_12075_b200 import build as tbn_build
from tests.head_util import reference, teacher_matrix

P = 0x10000          # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    tbn_build.build()
    return B.lib()


def xent_args(**kw):
    a = dict(x=P, w=P, dtype=B.BF16, T=4, d=64, V=100, bias=None, targets=P, ignore=-100, loss=P, lse=P, ws=P, nbytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def xent_bwd_args(**kw):
    a = dict(x=P, w=P, dtype=B.BF16, T=4, d=64, V=100, bias=None, targets=P, ignore=-100, lse=P, dloss=P, dx=P, dw=P, dw_dtype=B.BF16, db=None,
             ws=P, nbytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def distill_args(**kw):
    a = dict(x=P, w=P, dtype=B.BF16, T=4, d=64, V=100, bias=None, index=P, logit=P, top_dtype=B.F32, K=5, tau=1.0, loss=P, lse=P, ws=P,
             nbytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def distill_bwd_args(**kw):
    a = dict(x=P, w=P, dtype=B.BF16, T=4, d=64, V=100, bias=None, index=P, logit=P, top_dtype=B.F32, K=5, tau=1.0, lse=P, dloss=P, dx=P, dw=P,
             dw_dtype=B.BF16, db=None, ws=P, nbytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


COMMON = [(dict(x=None), -1), (dict(w=None), -1), (dict(dtype=7), -1), (dict(dtype=B.I32), -1), (dict(T=-1), -1), (dict(d=0), -1),
          (dict(V=0), -1), (dict(V=-5), -1), (dict(x=P + 2), -1), (dict(w=P + 8), -1), (dict(bias=P + 2), -1), (dict(ws=P + 4), -1),
          (dict(lse=None), -1), (dict(lse=P + 1), -1), (dict(ws=None), -4), (dict(nbytes=64), -4), (dict(T=1 << 31), -3),
          (dict(V=(1 << 31) - 1), -3)]


@pytest.mark.parametrize("change,status", COMMON + [(dict(targets=None), -1), (dict(targets=P + 4), -1), (dict(loss=None), -1)])
def test_xent_forward_refuses(lib, change, status):
    assert lib.tbn_linear_xent_fwd(*xent_args(**change)) == status


@pytest.mark.parametrize("change,status", COMMON + [(dict(dloss=None), -1), (dict(dx=P + 4), -1), (dict(dw=P + 4), -1), (dict(dw_dtype=2), -1),
                                                    (dict(db=P + 2), -1)])
def test_xent_backward_refuses(lib, change, status):
    assert lib.tbn_linear_xent_bwd(*xent_bwd_args(**change)) == status


DISTILL = [(dict(K=0), -1), (dict(K=-3), -1), (dict(K=1025), -3), (dict(tau=0.0), -1), (dict(tau=-1.0), -1), (dict(tau=math.nan), -1),
           (dict(tau=math.inf), -1), (dict(tau=1e-38), -1), (dict(index=None), -1), (dict(logit=None), -1), (dict(index=P + 4), -1),
           (dict(logit=P + 2), -1), (dict(top_dtype=2), -1)]


@pytest.mark.parametrize("change,status", COMMON + DISTILL)
def test_distill_forward_refuses(lib, change, status):
    assert lib.tbn_linear_distill_fwd(*distill_args(**change)) == status


@pytest.mark.parametrize("change,status", COMMON + DISTILL + [(dict(dloss=None), -1), (dict(dw_dtype=9), -1)])
def test_distill_backward_refuses(lib, change, status):
    assert lib.tbn_linear_distill_bwd(*distill_bwd_args(**change)) == status


def test_no_tokens_and_nothing_asked_for(lib):
    assert lib.tbn_linear_xent_fwd(*xent_args(T=0, x=None, loss=None, lse=None, ws=None, nbytes=0)) == 0
    assert lib.tbn_linear_distill_fwd(*distill_args(T=0, x=None, index=None, logit=None, ws=None, nbytes=0)) == 0
    assert lib.tbn_linear_xent_bwd(*xent_bwd_args(T=0, x=None, dw=None, db=None, ws=None, nbytes=0)) == 0
    assert lib.tbn_linear_xent_bwd(*xent_bwd_args(dx=None, dw=None, db=None)) == 0


def test_workspace_queries(lib):
    for dtype in (B.BF16, B.F32):
        fwd = lib.tbn_linear_xent_workspace_bytes(4096, 1024, 32768, dtype, 0)
        bwd = lib.tbn_linear_xent_workspace_bytes(4096, 1024, 32768, dtype, 1)
        logits = 4096 * 32768 * 4
        assert 0 < fwd < logits // 2 and 0 < bwd < 2 * logits
        # the piece of dz is bounded: a vocabulary twice as large does not need twice the room for it
        wide = lib.tbn_linear_xent_workspace_bytes(4096, 1024, 262144, dtype, 1)
        packed = 4 * 1024 * 262144 if dtype == B.F32 else 0
        assert wide - packed < bwd + (64 << 20)
        assert lib.tbn_linear_distill_workspace_bytes(4096, 1024, 32768, dtype, 64, 0) > fwd
    for bad in ((-1, 64, 100, B.BF16), (4, 0, 100, B.BF16), (4, 64, 0, B.BF16), (4, 64, 100, 5), (0, 64, 100, B.BF16)):
        assert lib.tbn_linear_xent_workspace_bytes(*bad, 0) == 0
        assert lib.tbn_linear_distill_workspace_bytes(*bad, 3, 1) == 0
    assert lib.tbn_linear_distill_workspace_bytes(4, 64, 100, B.BF16, 2000, 0) == 0


@pytest.mark.parametrize("T,V,K", [(1 << 27, 2**31 - 1025, 1), (2**31 - 1025, 2**31 - 1025, 1024), (1, 2**31 - 1025, 3), (2**31 - 1025, 1, 2)])
def test_distill_workspace_at_the_largest_sizes(lib, T, V, K):
    """The lists (8 bytes per entry) and the table of their starts (two entries of 2 bytes per token at least) are in it."""
    for dtype in (B.BF16, B.F32):
        for backward in (0, 1):
            rest = lib.tbn_linear_xent_workspace_bytes(T, 1, V, dtype, backward)
            assert lib.tbn_linear_distill_workspace_bytes(T, 1, V, dtype, K, backward) >= rest + T * (8 * K + 4)


def test_binding_checks_shapes_types_and_devices():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(10, 8, dtype=torch.bfloat16)
    t, f = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    idx, lg = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    with pytest.raises(B.TbnError):
        B.tbn_linear_xent_fwd(x, w[:, :4].contiguous(), t)
    with pytest.raises(TypeError):
        B.tbn_linear_xent_fwd(x, w.float(), t)
    with pytest.raises(B.TbnError):
        B.tbn_linear_xent_fwd(x, w, t[:3])
    with pytest.raises(B.TbnError):
        B.tbn_linear_xent_fwd(x, w, t.to(torch.int32))
    with pytest.raises(B.TbnError):
        B.tbn_linear_xent_fwd(x, w, t, bias=torch.zeros(9))
    with pytest.raises(B.TbnError):
        B.tbn_linear_xent_bwd(x, w, t, f[:2], f)
    with pytest.raises(B.TbnError):
        B.tbn_linear_distill_fwd(x, w, idx, lg[:, :2])
    with pytest.raises(B.TbnError):
        B.tbn_linear_distill_bwd(x, w, t, lg, f, f)
    with pytest.raises(ValueError):
        B.tbn_linear_xent_fwd(x, w, t)                       # tensors on the host


@pytest.mark.parametrize("K,tau", [(1, 1.0), (4, 2.0)])
def test_plain_form_gradients_match_differences(K, tau):
    g = torch.Generator().manual_seed(K)
    T, d, V = 4, 3, 7
    x, w, bias = torch.randn(T, d, generator=g).double(), torch.randn(V, d, generator=g).double(), torch.randn(V, generator=g).double()
    index, logit = torch.randint(-1, V, (T, K), generator=g), torch.randn(T, K, generator=g)
    index[2] = -1
    dloss = torch.rand(T, generator=g).double()
    dense = teacher_matrix(T, V, index, logit, tau)
    ref = reference(x, w, bias, dloss, tau, *dense)

    def total(x, w, bias):
        return float((reference(x, w, bias, dloss, tau, *dense)["loss"].cpu() * dloss).sum())

    h = 1e-5
    for name, grad, args in (("x", "dx", 0), ("w", "dw", 1), ("bias", "db", 2)):
        t = [x, w, bias][args]
        for i in range(t.numel()):
            up, down = [x.clone(), w.clone(), bias.clone()], [x.clone(), w.clone(), bias.clone()]
            up[args].view(-1)[i] += h
            down[args].view(-1)[i] -= h
            slope = (total(*up) - total(*down)) / (2 * h)
            # central differences: h^2 / 6 times a third derivative of order 10, and 1e-16 / h from the subtraction
            assert abs(slope - float(ref[grad].reshape(-1)[i])) < 1e-8, (name, i)
