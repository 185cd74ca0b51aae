"""The key/value cache's oracle against hand-made values and invariants."""
import math
from fractions import Fraction

import pytest
import torch

from oracle import kv


@pytest.mark.parametrize("largest", [1.0, 127.0, 65504.0, 6e-8, 0.3333, 1.9990234375, 3.3895e38, 127 * 4095 / 4096, 2.0 ** -90])
def test_scale_is_the_least_odd_number_of_12_bits(largest):
    s = Fraction(kv.scale_of(largest))
    unit = Fraction(2) ** (math.frexp(float(s))[1] - 12)
    assert (s / unit).denominator == 1 and (s / unit) % 2 == 1 and s / unit < 4096
    assert s >= Fraction(largest) / 127 or largest / 127 < 2.0 ** -100
    lower = s - 2 * unit if s / unit > 2049 else Fraction(4095, 2) * unit
    assert lower < max(Fraction(largest) / 127, Fraction(2) ** -100)


def test_scale_grows_with_its_argument_and_zero_has_one():
    values = [kv.scale_of(x) for x in sorted([0.0, 1e-30, 0.5, 0.50048828125, 1.0, 3.0, 64.0])]
    assert values == sorted(values) and values[0] > 0
    assert math.isnan(kv.scale_of(math.inf)) and math.isnan(kv.scale_of(math.nan))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_no_16_bit_number_is_half_way_between_two_codes(dtype):
    x = torch.randn(4096, generator=torch.Generator().manual_seed(1)).to(dtype).double()
    scale = kv.scale_of(float(x.abs().max()))
    middle = (x / scale - torch.floor(x / scale) - 0.5).abs()
    assert float(middle.min()) > 2.0 ** -21
    # so 32 bits decide as 64 do, also by the reciprocal
    inverse = torch.tensor(1.0, dtype=torch.float32) / torch.tensor(scale, dtype=torch.float32)
    assert torch.equal(torch.round(x.float() * inverse).long(), torch.round(x / scale).long())


def test_places_of_a_page():
    assert sorted(kv.PLACE) == list(range(64)) and kv.PLACE[:5] == [0, 1, 2, 3, 16] and kv.PLACE[16] == 4 and kv.PLACE[63] == 63


def test_attention_of_equal_keys_is_the_mean_of_the_values():
    codes = torch.full((1, 1, 2, 64, 64), 128, dtype=torch.uint8)
    for t in range(64):
        codes[0, 0, 1].view(-1, 64)[:, kv.PLACE[t]] = 128 + t
    scales = torch.tensor([[[1.0, 0.5]]])
    q = torch.ones((1, 1, 1, 64), dtype=torch.float16)
    out, lse, weights, *_ = kv.attention(codes, scales, torch.tensor([[0]]), [11], q, [1], 0.125, 0)
    assert torch.allclose(out, torch.full_like(out, 2.5)) and float(lse) == pytest.approx(math.log(11))
    assert torch.allclose(weights[0][0], torch.full((11,), 1 / 11, dtype=torch.float64))
    out, *_ = kv.attention(codes, scales, torch.tensor([[0]]), [11], q, [1], 0.125, 3)
    assert torch.allclose(out, torch.full_like(out, 4.5))


def test_choice_of_what_is_kept():
    w = torch.tensor([1.0, 5.0, 1.0, math.nan, 0.0, 1.0, 9.0, 0.0])
    assert kv.choose(w, 8, 4, 1) == [1, 3, 6, 7]
    assert kv.choose(w, 8, 5, 1) == [0, 1, 3, 6, 7]
    assert kv.choose(w, 8, 3, 3) == [5, 6, 7]
    assert kv.choose(w, 3, 5, 4) == [0, 1, 2]
    assert kv.choose(w, 0, 5, 4) == []
