"""8-bit products by every way through the kernels, with a bias: what a sum becomes is the header's steps, each rounded to fp32, bit for bit."""
import math

import pytest
import torch

from i8_paths import FEW, PATHS, pitch
from oracle import i8 as oracle
from test_gpu_i8 import gpu, guarded, rounded_to, same, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs_of(rows, N, K, seed=0):
    """codes, scales, weights, weight_scales, bias on the GPU; any codes, and anything behind a row's end."""
    gen = torch.Generator(device="cuda").manual_seed(seed + rows + N + K)

    def codes(n):
        return torch.randint(-128, 128, (n, pitch(K)), generator=gen, device="cuda", dtype=torch.int16).to(torch.int8)[:, :K]

    def normal(n):
        return torch.randn(n, generator=gen, device="cuda")

    c, w = codes(rows), codes(N)
    return c, torch.exp(normal(rows)) * 0.01, w, torch.exp(0.3 * normal(N)) * (0.02 / math.sqrt(K)), normal(N)


def by_steps(inputs):
    """fp32 [rows, N]: the exact sum, its rounding, the row's scale, the channel's, the bias: one rounding each."""
    codes, scales, weights, weight_scales, bias = inputs
    w = weights.double().t().contiguous()
    y = torch.empty((codes.shape[0], weights.shape[0]), device="cuda")
    for r in range(0, codes.shape[0], 1024):
        y[r : r + 1024] = torch.matmul(codes[r : r + 1024].double(), w).float()            # whole numbers under 2^53: exact, then rounded once
    y.mul_(scales[:, None])
    y.mul_(weight_scales)
    return y if bias is None else y.add_(bias)


def sixteens(gpu, inputs, dtype):  # noqa: F811
    """The gated product, sixteen rows at a time."""
    codes, scales, weights, weight_scales, bias = inputs
    y = torch.zeros((codes.shape[0], weights.shape[0] // 2), dtype=dtype, device="cuda")
    for r in range(0, codes.shape[0], 16):
        gpu.spqt_i8_gemm(codes[r : r + 16], scales[r : r + 16], weights, weight_scales, y[r : r + 16], bias=bias, gated=True)
    return y


def check_every_way(gpu, rows, N, K, dtype, biased=True):  # noqa: F811
    codes, scales, weights, weight_scales, bias = inputs = inputs_of(rows, N, K)
    if not biased:
        inputs = (*inputs[:4], None)
        bias = None
    space = gpu.new_i8_workspace(rows, N, K)
    space.fill_(255)
    want, gated = by_steps(inputs).to(dtype), sixteens(gpu, inputs, dtype)
    some = sorted({0, rows // 2, rows - 1})
    exact, off = oracle.product(codes[some].cpu(), scales[some].cpu(), weights.cpu(), weight_scales.cpu(), None if bias is None else bias.cpu(), gated=True)
    assert rounded_to(gated[some], exact, off, dtype)
    for given in (None, space):
        for result, is_gated in ((want, False), (gated, True)):
            n = result.shape[1]
            for pitch_y, at in ((n + 3, 1), (-(-n // 8) * 8, 0)):                            # rows that begin anywhere, and at 16 bytes
                y, whole = guarded(rows, n, pitch_y, dtype, at)
                gpu.spqt_i8_gemm(codes, scales, weights, weight_scales, y, bias=bias, gated=is_gated, workspace=given)
                assert same(y, result), (is_gated, given is not None, (y != result).nonzero()[:3].tolist())
                assert untouched(y, whole)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,N,K", FEW + list(PATHS.values()), ids=lambda v: str(v))
def test_every_step_is_rounded_whichever_way(gpu, rows, N, K, dtype):  # noqa: F811
    check_every_way(gpu, rows, N, K, getattr(torch, dtype))
