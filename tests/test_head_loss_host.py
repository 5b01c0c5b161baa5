"""What a head-loss call costs before anything runs on the GPU: workspace and host time."""
import time

import pytest

from paper_2407_12075_b200 import binding as B
from paper_2407_12075_b200 import build as tbn_build


@pytest.fixture(scope="module")
def lib():
    tbn_build.build()
    return B.lib()


@pytest.mark.parametrize("T,d,V,dtype", [(2100, 64, 9001, B.BF16), (8192, 64, 131072, B.BF16), (4096, 128, 100000, B.BF16), (333, 768, 10007, B.BF16),
                                         (777, 501, 4999, B.F32), (1, 64, 500000, B.F32), (100000, 2048, 1000, B.BF16)])
def test_planning_a_backward_takes_little_host_time(lib, T, d, V, dtype):
    """The splits of the two gradient products are chosen anew in every call: microseconds, beside a launch's two or three."""
    best = 1.0
    for _ in range(300):
        t0 = time.perf_counter()
        lib.tbn_linear_xent_workspace_bytes(T, d, V, dtype, 1)
        best = min(best, time.perf_counter() - t0)
    assert best < 20e-6, best


def test_packed_weights_of_the_backward_are_bounded(lib):
    """Weights that cannot be read in place are packed for one piece of the vocabulary at a time."""
    T = 4096
    for dtype, d in ((B.F32, 1024), (B.BF16, 1001)):
        small, large = (lib.tbn_linear_xent_workspace_bytes(T, d, V, dtype, 1) for V in (1 << 18, 1 << 21))
        assert large < small + (128 << 20)


def test_partial_statistics_are_small_beside_the_logits(lib):
    """One record of 16 bytes per token and 64 classes or more: a sixteenth of the fp32 logits (and the small packed operands)."""
    for dtype in (B.BF16, B.F32):
        T, d, V = 8192, 64, 131072
        assert lib.tbn_linear_xent_workspace_bytes(T, d, V, dtype, 0) < T * V * 4 / 15 + 6 * (T + V) * d


def test_operands_whose_byte_counts_would_wrap_are_refused(lib):
    top, P = 2**31 - 1025, 0x10000                       # P: never dereferenced
    for T, d, V in ((top, top, top), (4, top, top), (top, 2049, 4)):
        for dtype in (B.BF16, B.F32):
            assert lib.tbn_linear_xent_workspace_bytes(T, d, V, dtype, 1) == 0
            assert lib.tbn_linear_xent_fwd(P, P, dtype, T, d, V, None, P, -100, P, P, P, 1 << 62, None) == -3
            assert lib.tbn_linear_distill_bwd(P, P, dtype, T, d, V, None, P, P, B.F32, 3, 1.0, P, P, P, P, dtype, None, P, 1 << 62, None) == -3
    assert lib.tbn_linear_xent_workspace_bytes(top, 1, top, B.F32, 1) > 0
