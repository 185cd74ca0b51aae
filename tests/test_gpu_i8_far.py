"""8-bit products by tiles whose rows are so far apart that places pass 2^31, up to the strides that the tiles take and just behind them."""
import pytest
import torch

from i8_paths import FAR
from test_gpu_i8 import gpu, same  # noqa: F401
from test_gpu_i8_ways import by_steps, inputs_of, sixteens

pytestmark = pytest.mark.gpu


def apart(t, stride):
    """t with rows that begin `stride` elements apart."""
    if stride == t.stride(0):
        return t
    whole = torch.empty(t.shape[0] * stride, dtype=t.dtype, device="cuda")
    there = whole.view(t.shape[0], stride)[:, : t.shape[1]]
    there.copy_(t)
    return there


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,N,K,gated,codes_row,weights_row,y_row,tile", FAR)
def test_products_of_rows_far_apart(gpu, rows, N, K, gated, codes_row, weights_row, y_row, tile, dtype):  # noqa: F811
    dtype = getattr(torch, dtype)
    inputs = inputs_of(rows, N, K)
    want = sixteens(gpu, inputs, dtype) if gated else by_steps(inputs).to(dtype)
    codes, weights = apart(inputs[0], codes_row), apart(inputs[2], weights_row)
    assert codes.stride(0) == codes_row and weights.stride(0) == weights_row
    whole = torch.full((rows, y_row), 7.0, dtype=dtype, device="cuda")
    y = whole[:, : want.shape[1]]
    gpu.spqt_i8_gemm(codes, inputs[1], weights, inputs[3], y, bias=inputs[4], gated=gated)
    assert same(y.contiguous(), want)
    y.fill_(7.0)
    assert all(bool((part == 7).all()) for part in whole.split(64))
