"""Norms of 8-bit integers' prompt side at the edges of what a call may ask for, against 64 bits."""
import pytest
import torch

from oracle import i8 as oracle
from test_gpu_i8 import gpu, rounded_to  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [2.0**-99, 1.0, 2.0**100, 2.0**126, 2.0**127])
@pytest.mark.parametrize("K", [3, 64, 1000, 3001, 9001, 20000, 40000])
def test_norms_with_any_eps(gpu, K, eps):  # noqa: F811
    """eps is any number of fp32 from 1e-30 on, next to rows of any size: in both norms, alone and together with a block."""
    dtype = torch.bfloat16
    gen = torch.Generator().manual_seed(K)

    def normal(*shape):
        return torch.randn(shape, generator=gen)

    h = normal(9, K) * (2.0 ** torch.tensor([-60.0, 0.0, 20.0, 50.0, 60.0, 63.0, 64.0, 100.0, 0.0]))[:, None]
    h[8] = 0
    h = h.to(dtype)
    gain = (2.0**40 * normal(K)).to(dtype)
    out, scales = torch.zeros((9, K), dtype=dtype, device="cuda"), torch.zeros(9, device="cuda")
    codes = gpu.new_i8_codes(9, K)
    gpu.spqt_i8_norm(h.cuda(), gain.cuda(), eps=eps, out=out, codes=codes, scales=scales)
    least = 2.0**-149                                     # what a step of subnormal numbers on the way may be off by
    _, x, _, far = oracle.norm(h.double(), gain.double(), eps=eps)
    far = far + gain.double().abs() * least
    assert rounded_to(out, x, far, dtype)
    top = x.abs().max(dim=1)[0].clamp(min=2.0**-100)
    assert bool(((scales.double().cpu() * 127 - top).abs() <= far.max(dim=1)[0] + 2 * oracle.U * top).all())

    def inverse(v):
        return 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + eps)

    block, zero = h.flip(0), torch.zeros_like(h)
    h_out = torch.zeros_like(out)
    gpu.spqt_i8_norm(zero.cuda(), gain.cuda(), block=block.cuda(), block_gain=gain.cuda(), eps=eps, h_out=h_out, out=out)
    s, x, off, far = oracle.norm(zero.double(), gain.double(), block=block.double(), block_gain=gain.double(), eps=eps)
    first = block.double() * inverse(block.double())
    moved = torch.where(first.abs() < 2.0**-125, gain.double().abs() * least, torch.zeros_like(first))
    assert rounded_to(h_out, s, off + moved, dtype)
    by = inverse(s)
    far = far + moved * by * gain.double().abs() + x.abs() * torch.sqrt((moved * moved).mean(dim=1, keepdim=True)) * by + gain.double().abs() * least
    assert rounded_to(out, x, far, dtype)


@pytest.mark.parametrize("K", [7, 512, 4096, 20000, 65536])
def test_only_a_subnormal_reciprocal_loses_digits(gpu, K):  # noqa: F811
    """Rows summed in units of 2^80 are as exact as others; where 1 / RMS is a subnormal number, half a step of 2^-149 comes on top."""
    dtype = torch.bfloat16
    gen = torch.Generator().manual_seed(K)
    size = torch.tensor([2.0**56, 2.0**60, 2.0**64, 2.0**100, 2.0**124, 2.0**127])[:, None]
    h = (size * (0.5 + 0.5 * torch.rand((6, K), generator=gen))).to(dtype)
    h[5] = torch.finfo(dtype).max
    h[:, ::3] *= -1
    gain = torch.randn(K, generator=gen).to(dtype)
    out, codes, scales = torch.zeros((6, K), dtype=dtype, device="cuda"), gpu.new_i8_codes(6, K), torch.zeros(6, device="cuda")
    gpu.spqt_i8_norm(h.cuda(), gain.cuda(), out=out, codes=codes, scales=scales)
    _, x, _, far = oracle.norm(h.double(), gain.double())
    far[5] += x[5].abs() * 2.0**-150 * 2.0**128
    assert rounded_to(out, x, far, dtype)
    top = x.abs().max(dim=1)[0]
    assert bool(((scales.double().cpu() * 127 - top).abs() <= far.max(dim=1)[0] + 2 * oracle.U * top).all())
