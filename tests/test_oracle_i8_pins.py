"""The oracle of the prompt side in 8-bit integers against hand-made values and invariants."""
import math

import pytest
import torch

from oracle import i8


def test_codes_of_simple_rows():
    x = torch.tensor([[1.27, -0.64, 0.0, 0.005, 0.006], [0, 0, 0, 0, 0], [math.inf, 1, 2, 3, 4], [1, math.nan, 0, 0, 0], [2, 1, -1, -2, 0]], dtype=torch.float16)
    codes, scales = i8.quantize(x)
    assert codes[0].tolist() == [127, -64, 0, 1, 1] and codes[1].tolist() == [0] * 5 and codes[2].tolist() == [0] * 5 and codes[3].tolist() == [0] * 5
    assert codes[4].tolist() == [127, 64, -64, -127, 0]          # half of the largest is 63.5: to the even neighbour
    assert scales[2].isnan() and scales[3].isnan() and float(scales[4]) == pytest.approx(2 / 127, rel=2.0 ** -24)
    assert float(scales[1]) > 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_codes_stand_for_is_half_a_scale_away_at_most(dtype):
    x = torch.randn((20, 300), generator=torch.Generator().manual_seed(1)).to(dtype)
    codes, scales = i8.quantize(x)
    assert int(codes.abs().max()) == 127
    back = i8.read(codes, scales, dtype).double()
    assert bool(((back - x.double()).abs() <= scales.double()[:, None] * 0.5 * (1 + 2.0 ** -15) + back.abs() * i8.half_step(dtype)).all())


def test_reading_stays_within_the_type():
    x = torch.tensor([[65504.0, -65504.0, 1.0]], dtype=torch.float16)
    assert i8.read(*i8.quantize(x), torch.float16)[0].tolist() == [65504.0, -65504.0, 0.0]


def test_a_norm_by_hand():
    h, gain = torch.tensor([[3.0, 4.0]], dtype=torch.float64), torch.tensor([1.0, 2.0], dtype=torch.float64)
    s, x, off, far = i8.norm(h, gain, eps=1e-9)
    r = math.sqrt(12.5)
    assert torch.allclose(x, torch.tensor([[3 / r, 8 / r]], dtype=torch.float64)) and torch.equal(s, h) and float(off.abs().max()) == 0
    s, x, off, far = i8.norm(h, gain, block=h, block_gain=gain, gate=gain, residual=0.5, offset=1.0, eps=1e-9)
    z = torch.tensor([[3 / r * 2, 4 / r * 3 * 2]], dtype=torch.float64)
    assert torch.allclose(s, 0.5 * h + z)
    assert torch.allclose(x, s / s.pow(2).mean().sqrt() * (1 + gain))
    assert bool((off > 0).all()) and bool((far > 0).all()) and float((far / x.abs()).max()) < 1e-5


def test_fp32_steps_stay_within_the_norms_bound():
    gen = torch.Generator().manual_seed(2)
    h, block, gain = torch.randn((30, 900), generator=gen), torch.randn((30, 900), generator=gen), 1 + 0.1 * torch.randn(900, generator=gen)
    s, x, off, far = i8.norm(h.double(), gain.double(), block=block.double(), block_gain=gain.double())
    z = block * (1 / torch.sqrt((block * block).mean(1, keepdim=True) + 1e-5)) * gain
    t = h + z
    u = t * (1 / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-5)) * gain
    assert bool(((t.double() - s).abs() <= off).all()) and bool(((u.double() - x).abs() <= far).all())


def test_products_by_hand():
    codes, weights = torch.tensor([[1, 2], [-3, 4]], dtype=torch.int8), torch.tensor([[5, 6], [7, -8]], dtype=torch.int8)
    a, w = torch.tensor([0.5, 2.0]), torch.tensor([1.0, 0.25])
    y, off = i8.product(codes, a, weights, w, bias=torch.tensor([1.0, 0.0]))
    assert y.tolist() == [[17 * 0.5 + 1, -9 * 0.5 * 0.25], [9 * 2 + 1, -53 * 2 * 0.25]]
    assert bool((off > 0).all()) and float((off / y.abs()).max()) < 1e-6
    y, _ = i8.product(codes, a, weights, w, gated=True)
    assert float(y[0, 0]) == pytest.approx(8.5 / (1 + math.exp(-8.5)) * -1.125)
