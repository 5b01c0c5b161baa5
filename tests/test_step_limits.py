"""Embedding, LayerNorm for training and head losses: the largest sizes that the header allows, and the first ones beyond them."""
import pytest

from paper_2407_12075_b200 import binding as B
from paper_2407_12075_b200 import build as tbn_build

P = 0x10000                                                              # never dereferenced
MOST, WIDEST = 2 ** 31 - 1025, 2 ** 23


@pytest.fixture(scope="module")
def lib():
    tbn_build.build()
    return B.lib()


def test_the_last_sizes_have_a_workspace(lib):
    assert lib.tbn_embedding_bwd_workspace_bytes(MOST, 1, MOST) > 0
    assert lib.tbn_embedding_bwd_workspace_bytes(4, WIDEST, 100) > 0
    assert lib.tbn_layernorm_bwd_workspace_bytes(MOST, 1) > 0 and lib.tbn_layernorm_bwd_workspace_bytes(4, WIDEST) > 0
    assert lib.tbn_embedding_bwd_workspace_bytes(MOST + 1, 1, 100) == lib.tbn_embedding_bwd_workspace_bytes(4, 1, MOST + 1) == 0
    assert lib.tbn_embedding_bwd_workspace_bytes(4, WIDEST + 1, 100) == 0
    assert lib.tbn_layernorm_bwd_workspace_bytes(MOST + 1, 1) == lib.tbn_layernorm_bwd_workspace_bytes(4, WIDEST + 1) == 0


@pytest.mark.parametrize("T,vocab,d", [(MOST + 1, 100, 8), (4, MOST + 1, 8), (4, 100, WIDEST + 1)])
def test_embedding_beyond(lib, T, vocab, d):
    assert lib.tbn_embedding_fwd(P, T, P, B.BF16, vocab, d, -1, 1.0, P, B.BF16, None) == -3
    assert lib.tbn_embedding_tiled_fwd(P, T, vocab, d, P, 1, P, B.ALPHA_PER_TILE, -1, 1.0, P, B.BF16, None) == -3
    assert lib.tbn_embedding_bwd(P, T, P, B.BF16, vocab, d, -1, 1.0, P, B.F32, 0, P, 1 << 62, None) == -3


@pytest.mark.parametrize("T,d", [(MOST + 1, 8), (4, WIDEST + 1)])
def test_layernorm_beyond(lib, T, d):
    assert lib.tbn_layernorm_train_fwd(P, None, B.BF16, T, d, P, P, 1e-5, None, P, B.BF16, P, P, None) == -3
    assert lib.tbn_layernorm_bwd(P, B.BF16, P, B.BF16, T, d, P, P, P, None, P, P, P, P, 1 << 62, None) == -3


def test_head_loss_beyond(lib):
    for backward in (0, 1):
        assert lib.tbn_linear_xent_workspace_bytes(MOST, 8, 8, B.BF16, backward) > 0
        assert lib.tbn_linear_xent_workspace_bytes(MOST + 1, 8, 8, B.BF16, backward) == lib.tbn_linear_xent_workspace_bytes(8, 8, MOST + 1, B.BF16, backward) == 0
