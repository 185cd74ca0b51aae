"""Gated 8-bit products whose gates saturate: every way through the kernels against the formula in 64 bits."""
import math

import pytest
import torch

from i8_paths import FEW, PATHS, pitch
from oracle import i8 as oracle

U = oracle.U
# Where 1 + exp(-gate) is a number of fp32 whose reciprocal is not a normal one (-87.34 to -88.72), and all around it.
GATES = [-0.5, -20.0, -86.0, -87.25, -87.375, -87.75, -88.0, -88.5, -88.71875, -88.75, -89.5, -91.0, -100.0, -200.0, -1e38, -math.inf, math.nan, math.inf, 0.0, 1e-38, 3.0, 90.0, 3e38]
UPS = [1.0, -3.0, 2.0**60, -(2.0**118), 2.0**-60]         # times the gate


def bounds(dtype):
    """The formula of each gate and up, and how far fp32 steps may be from it: [gates, ups] twice."""
    g32 = torch.tensor(GATES)[:, None]
    u = (g32 * torch.tensor(UPS)).double()
    g = g32.double()
    y = g * torch.sigmoid(g) * u
    # Halves of fp32's steps. 32 bits: the hardware's power and reciprocal (2 each), the factor beside the power, the sum, and two products: 8; where the reciprocal is a subnormal
    # number, of 2^-128 and more, half a step of 2^-149 is 4 of them. 16 bits: the power's argument is off by 1.3 |g| + 3, power and reciprocal by 2 each, a sum and three products by 4.
    # Steps of subnormal numbers on the way are 2^-149.
    steps = torch.where(g < -87.3, 12.0, 8.0).double() if dtype == torch.float32 else 1.3 * g.abs().clamp(max=100.0) + 11.0
    off = y.abs() * steps * U * 1.001 + (g.abs().clamp(max=100.0) + 1.0) * 2.0**-149 * (1.0 + u.abs().clamp(max=2.0**128))
    off = torch.where(y.isinf(), torch.zeros_like(off), off)
    low, high = y - off, y + off
    gone = (g < -88.72) & torch.isfinite(y)               # 1 + exp(-gate) leaves fp32: the quotient is 0, or what it is
    low, high = torch.where(gone, torch.minimum(low, -off), low), torch.where(gone, torch.maximum(high, off), high)
    return y, low, high


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,N,K", FEW + list(PATHS.values()), ids=lambda v: str(v))
def test_gates_that_saturate(rows, N, K, dtype):
    import paper_2511_04477_amd as spqt
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.randint(-127, 128, (rows, pitch(K)), generator=gen, device="cuda", dtype=torch.int32).to(torch.int8)[:, :K]
    weights = torch.zeros((N, pitch(K)), dtype=torch.int8, device="cuda")[:, :K]
    at = K // 3                                           # sums are 1: a product is a row's scale times a channel's
    codes[:, at] = 1
    weights[:, at] = 1
    row, column = torch.arange(rows) % len(GATES), torch.arange(N // 2) % len(UPS)
    scales = torch.tensor(GATES)[row].cuda()
    weight_scales = torch.cat([torch.ones(N // 2), torch.tensor(UPS)[column]]).cuda()
    _, low, high = bounds(dtype)
    low, high = low.to(dtype)[row].cuda()[:, column.cuda()].float(), high.to(dtype)[row].cuda()[:, column.cuda()].float()     # rounding keeps their order
    for space in (None, spqt.new_i8_workspace(rows, N, K)):
        y = torch.full((rows, N // 2), 7.0, dtype=dtype, device="cuda")
        spqt.spqt_i8_gemm(codes, scales, weights, weight_scales, y, gated=True, workspace=space)
        v = y.float()
        right = torch.where(low.isnan(), v.isnan(), (v >= low) & (v <= high))
        wrong = (~right).nonzero()[:3].tolist()
        assert not wrong, [(GATES[r % len(GATES)], UPS[c % len(UPS)], v[r, c].item(), low[r, c].item(), high[r, c].item()) for r, c in wrong]


def test_the_bounds_tell_zero_from_the_formula():
    """Where the quotient is a number of fp32, outputs of 0 are outside the bounds for some up, in every type."""
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        _, low, high = bounds(dtype)
        low, high = low.to(dtype), high.to(dtype)
        for i, g in enumerate(GATES):
            if -88.72 < g < -0.1:
                assert bool(((low[i] > 0) | (high[i] < 0)).any()), (dtype, g)
