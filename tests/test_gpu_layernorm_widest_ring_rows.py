"""Rows about the widths from which on they no longer fit a thread block's registers, 1024 pieces of eight columns: 8192 columns, 8188 where
rows begin up to 4 columns inside a piece, 8186 with up to 6, 8185 with up to 7; and rows whose last piece the shift decides on."""
import pytest

from tests import test_gpu_layernorm_train as ordinary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d", [(3, 8176), (9, 8183), (3, 8184), (17, 8185), (9, 8186), (9, 8187), (5, 8188), (9, 8190), (9, 8191), (3, 8193),
                                 (70, 28), (70, 27), (70, 26), (70, 25), (300, 60), (300, 124), (40, 252), (40, 253), (20, 508), (20, 1020), (20, 1022), (9, 4092)])
@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("residual,affine", [(False, True), (True, True), (True, False)])
def test_forward_and_backward(T, d, x_dtype, y_dtype, residual, affine):
    ordinary.test_forward_and_backward(T, d, x_dtype, y_dtype, residual, affine)
