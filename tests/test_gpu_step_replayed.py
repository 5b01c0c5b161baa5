"""Captured calls of every size class, replayed with other inputs in the same tensors; calls that share a workspace one after another."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B
from tests.test_gpu_embedding import rand, some_ids

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def replayed(call, inputs, fresh):
    """call(*inputs) captured, then replayed with the values of each of `fresh`: equal to the eager call's bits."""
    first = [t.clone() for t in inputs]
    call(*first)                                                        # the library's one-time settings are made outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(*inputs)
    for values in fresh:
        for t, v in zip(inputs, values):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        want = call(*values)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("T,V,d", [(300, 50, 257), (8192, 700, 64), (20_000, 70_000, 24), (12_000, 2 ** 20 + 5, 9), (40_000, 1000, 501)])
@pytest.mark.parametrize("add", [False, True])
def test_embedding(T, V, d, add):
    ws = torch.empty(B.tbn_embedding_bwd_workspace_bytes(T, d, V), dtype=torch.uint8, device=DEV)

    def call(ids, dy, table, dw):
        y = B.tbn_embedding_fwd(ids, table, 2.0)
        a = B.tbn_embedding_bwd(ids, dy, V, 0.5, add_to=dw.clone() if add else None, workspace=ws)
        b = B.tbn_embedding_bwd(ids.flip(0), dy, V, 0.5, workspace=ws)          # the same workspace again
        return y, a, b
    make = lambda s, kind: (some_ids(s, T, V, kind), rand(s + 1, T, d), rand(s + 2, V, d), rand(s + 3, V, d))  # noqa: E731
    replayed(call, make(500, "even"), [make(510, "skewed"), make(520, "few"), make(530, "last")])


@pytest.mark.parametrize("T,d", [(16, 512), (777, 501), (3000, 100), (5000, 2048), (40, 8187), (20, 9001)])
def test_layernorm(T, d):
    ws = torch.empty(max(1, B.tbn_layernorm_bwd_workspace_bytes(T, d)), dtype=torch.uint8, device=DEV)

    def call(x, r, dy):
        y, s, mean, rstd = B.tbn_layernorm_train_fwd(x, residual=r)
        return (y, s, *B.tbn_layernorm_bwd(dy, s, mean, rstd, dsum=r, workspace=ws), *B.tbn_layernorm_bwd(r, s, mean, rstd, workspace=ws))
    make = lambda s: tuple(rand(s + i, T, d, dtype=torch.bfloat16) for i in range(3))  # noqa: E731
    replayed(call, make(600), [make(610), make(620)])
