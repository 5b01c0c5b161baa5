"""Embedding, LayerNorm for training and AdamW: what the entry points refuse, on the host and before anything is launched."""
import ctypes

import pytest
import torch

from paper_2407_12075_b200 import binding as B
from paper_2407_12075_b200 import build as tbn_build

P = 0x10000                                                              # never dereferenced
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    tbn_build.build()
    return B.lib()


def refused(call, args, changes):
    for index, value, status in changes:
        bad = list(args)
        bad[index] = value
        assert call(*bad) == status, (index, value)


def test_embedding(lib):
    args = [P, 4, P, B.BF16, 100, 64, -1, 1.0, P, B.BF16, None]
    refused(lib.tbn_embedding_fwd, args, [(0, None, -1), (0, P + 4, -1), (1, -1, -1), (1, 1 << 31, -3), (2, None, -1), (2, P + 8, -1), (3, 2, -1),
                                          (4, 0, -1), (4, 2**31 - 1, -3), (5, 0, -1), (5, 1 << 24, -3), (8, None, -1), (8, P + 2, -1), (9, 5, -1)])
    args = [P, 4, 100, 64, P, 4, P, B.ALPHA_PER_TILE, -1, 1.0, P, B.BF16, None]
    refused(lib.tbn_embedding_tiled_fwd, args, [(0, None, -1), (4, None, -1), (4, P + 4, -1), (5, 0, -1), (5, 7, -2), (6, None, -1), (6, P + 2, -1),
                                                (7, 2, -1), (10, None, -1), (11, 2, -1)])
    args = [P, 4, P, B.BF16, 100, 64, -1, 1.0, P, B.F32, 0, P, 1 << 30, None]
    refused(lib.tbn_embedding_bwd, args, [(0, None, -1), (1, -1, -1), (2, None, -1), (3, 2, -1), (4, -5, -1), (5, 1 << 24, -3), (8, None, -1),
                                          (8, P + 4, -1), (9, 2, -1), (11, None, -4), (11, P + 8, -4), (12, 100, -4)])
    assert lib.tbn_embedding_bwd_workspace_bytes(4, 64, 100) > 0
    assert lib.tbn_embedding_bwd_workspace_bytes(0, 64, 100) == lib.tbn_embedding_bwd_workspace_bytes(4, -1, 100) == 0


def test_layernorm(lib):
    args = [P, P, B.BF16, 4, 64, P, P, 1e-5, P, P, B.BF16, P, P, None]
    refused(lib.tbn_layernorm_train_fwd, args, [(0, None, -1), (0, P + 2, -1), (1, P + 2, -1), (2, 2, -1), (3, -1, -1), (3, 1 << 31, -3), (4, 0, -1),
                                                (4, 1 << 24, -3), (5, P + 1, -1), (6, P + 2, -1), (7, -1.0, -1), (7, NAN, -1), (8, None, -1),
                                                (8, P + 8, -1), (9, None, -1), (10, 2, -1), (11, P + 2, -1), (12, P + 1, -1)])
    args = [P, B.BF16, P, B.BF16, 400, 64, P, P, P, P, P, P, P, P, 1 << 30, None]
    refused(lib.tbn_layernorm_bwd, args, [(0, None, -1), (0, P + 2, -1), (1, 2, -1), (2, None, -1), (3, 9, -1), (4, -1, -1), (4, 1 << 31, -3), (5, 0, -1),
                                          (6, P + 2, -1), (7, None, -1), (8, None, -1), (9, P + 4, -1), (10, None, -1), (11, P + 1, -1), (12, P + 2, -1),
                                          (13, None, -4), (13, P + 4, -1), (14, 64, -4)])
    assert lib.tbn_layernorm_bwd_workspace_bytes(400, 64) > 0 and lib.tbn_layernorm_bwd_workspace_bytes(0, 64) == 0


def tensor(**changes):
    t = B._AdamWTensor(P, P, P, P, P, P, P, 1000, 0.1, B.F32, B.BF16, 8)
    for name, value in changes.items():
        setattr(t, name, value)
    return t


BAD_TENSORS = [(dict(param=None), -1), (dict(param=P + 2), -1), (dict(grad=None), -1), (dict(grad=P + 1), -1), (dict(m=None), -1), (dict(v=None), -1),
               (dict(m_scale=None), -1), (dict(v_scale=P + 2), -1), (dict(copy=P + 1), -1), (dict(n=-1), -1), (dict(n=1 << 43), -3),
               (dict(weight_decay=NAN), -1), (dict(weight_decay=INF), -1), (dict(param_dtype=2), -1), (dict(grad_dtype=-1), -1), (dict(state_bits=4), -1),
               (dict(state_bits=32, m=P + 2), -1)]


@pytest.mark.parametrize("place", [0, 1])
def test_adamw_tensors(lib, place):
    for changes, status in BAD_TENSORS:
        table = (B._AdamWTensor * 2)(tensor(), tensor())
        table[place] = tensor(**changes)
        assert lib.tbn_adamw_step(ctypes.addressof(table), 2, 1, None, 1e-3, None, 0.9, 0.999, 1e-8, None, 0, None) == status, changes


def test_adamw_arguments(lib):
    table = (B._AdamWTensor * 1)(tensor())
    args = [ctypes.addressof(table), 1, 1, None, 1e-3, None, 0.9, 0.999, 1e-8, None, 0, None]
    refused(lib.tbn_adamw_step, args, [(0, None, -1), (1, -1, -1), (2, 0, -1), (3, P + 4, -1), (4, NAN, -1), (4, INF, -1), (5, P + 1, -1), (6, 1.0, -1),
                                       (6, -0.1, -1), (6, NAN, -1), (7, 1.5, -1), (8, 0.0, -1), (8, NAN, -1), (9, P + 2, -1)])
    assert lib.tbn_adamw_step(None, 0, 1, None, 1e-3, None, 0.9, 0.999, 1e-8, None, 0, None) == 0
    args = [ctypes.addressof(table), 1, 1.0, P, P, P, 1 << 30, None]
    refused(lib.tbn_grad_norm, args, [(0, None, -1), (1, -1, -1), (2, 0.0, -1), (2, NAN, -1), (3, P + 2, -1), (4, P + 1, -1), (5, None, -4), (5, P + 8, -4),
                                      (6, 8, -4)])
    outs = (ctypes.c_void_p * 1)(P + 2)
    assert lib.tbn_adamw_unpack(ctypes.addressof(table), 1, ctypes.addressof(outs), None, None) == -1
    table[0].state_bits = 32
    assert lib.tbn_adamw_unpack(ctypes.addressof(table), 1, None, None, None) == -1


def test_tensors_on_the_cpu_are_refused(lib):
    x, ids, ones = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64), torch.ones(4)
    with pytest.raises(ValueError):
        B.tbn_embedding_fwd(ids, x)
    with pytest.raises(ValueError):
        B.tbn_embedding_bwd(ids, x, 10)
    with pytest.raises(ValueError):
        B.tbn_layernorm_train_fwd(x)
    with pytest.raises(ValueError):
        B.tbn_layernorm_bwd(x, x, ones, ones)
    with pytest.raises(ValueError):
        B.tbn_adamw_tensors([x], [x], [x], [x])


def test_sizes_and_types_that_do_not_fit(lib):
    ids, x = torch.zeros(4, dtype=torch.int64), torch.zeros(4, 64)
    with pytest.raises(TypeError):
        B.tbn_embedding_fwd(ids.int(), x)
    with pytest.raises(B.TbnError):
        B.tbn_embedding_fwd(ids, x[0])
    with pytest.raises(B.TbnError):
        B.tbn_embedding_bwd(ids[:3], x, 10)
    with pytest.raises(B.TbnError):
        B.tbn_adamw_tensors([x], [x], [x, x], [x])
    with pytest.raises(ValueError):
        B.tbn_adamw_state([x], bits=4)
    m, v, ms, vs = B.tbn_adamw_state([torch.zeros(257), torch.zeros(0)], 8)
    assert [t.numel() for t in m] == [t.numel() for t in v] == [257, 0] and [t.numel() for t in ms] == [t.numel() for t in vs] == [2, 0]
