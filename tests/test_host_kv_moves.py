"""What the exact eviction makes of a block's codes, on the CPU: the oracle's rule and what follows from it."""
import ctypes
import math

import pytest
import torch

import paper_2511_04477_amd as spqt
from oracle import kv
from test_host_kv import EINVAL, ESHAPE, ESIZE, attention, cache, rows


def block(seed, dtype=torch.float16, tokens=64, dim=128, size=1.0):
    x = (size * torch.randn(tokens, dim, generator=torch.Generator().manual_seed(seed))).to(dtype)
    return kv.quantize(x.double())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_block_that_stays_whole_stays_as_it_is(dtype):
    for seed in range(200):
        codes, scale = block(seed, dtype, dim=16, size=math.exp(seed % 7 - 3))
        again, same = kv.requantize([(codes, scale)])
        assert same == scale and torch.equal(again, codes)


def test_by_way_of_fp16_it_grows():
    """What the exact way is for: the scale after 50 moves as values read back in 16 bits."""
    growth = []
    for seed in range(30):
        codes, first = block(seed)
        scale = first
        for _ in range(50):
            codes, scale = kv.quantize(kv.rounded(codes.double() * scale, torch.float16).double())
        growth.append(scale / first - 1)
    assert min(growth) >= 0 and 0.003 < sum(growth) / len(growth) < 0.03


def test_blocks_that_come_together():
    """No value is further off than half of the new step, and codes stay within 127."""
    for seed in range(100):
        parts = [block(seed + 1000 * i, tokens=n, dim=32, size=s) for i, (n, s) in enumerate(((20, 1.0), (30, 0.3 + seed % 5), (14, 1e-3)))]
        codes, scale = kv.requantize(parts)
        before = torch.cat([c.double() * s for c, s in parts])
        assert int(codes.abs().max()) == 127
        # (the quotient of the scales is rounded to 32 bits)
        assert float((codes.double() * scale - before).abs().max()) <= scale * (0.5 + 127 * 2.0 ** -24)
        again, same = kv.requantize([(codes, scale)])
        assert same == scale and torch.equal(again, codes)


def test_zeros_and_no_numbers():
    zero = (torch.zeros((5, 8), dtype=torch.long), 3.0)
    codes, scale = kv.requantize([zero, (torch.zeros((2, 8), dtype=torch.long), 2.0 ** -99)])
    assert int(codes.abs().max()) == 0 and scale == kv.scale_of(0.0)
    codes, _ = kv.requantize([zero, (torch.full((1, 8), 127), kv.scale_of(1e-20))])
    assert torch.equal(codes[:5], zero[0]) and int(codes[5:].min()) == 127
    assert math.isnan(kv.requantize([zero, (torch.zeros((1, 8), dtype=torch.long), math.nan)])[1])


def test_refusals_are_those_of_the_other_eviction():
    evict = spqt.lib().spqt_kv_evict_exact
    whole = cache(weights=1 << 20)
    for args, status in (((0, 0, 1 << 21, 2, 1 << 21, 1 << 20), EINVAL), ((64, 65, 1 << 21, 2, 1 << 21, 1 << 20), EINVAL), ((129, 1, 1 << 21, 2, 1 << 21, 1 << 20), ESHAPE),
                         ((64, 1, None, 2, 1 << 21, 1 << 20), EINVAL)):
        assert evict(ctypes.byref(whole), *args, None) == status
    assert evict(ctypes.byref(cache()), 64, 1, 1 << 21, 2, 1 << 21, 1 << 20, None) == EINVAL


def test_outputs_over_the_queries_that_the_weights_need():
    weighed = dict(lse=1 << 22, size=16)                     # (a workspace that is too small: nothing is launched)
    assert attention(cache(weights=1 << 20), rows(), rows(), **weighed) == EINVAL
    assert attention(cache(weights=1 << 20), rows(), rows(data=1 << 21), **weighed) == ESIZE
    assert attention(cache(), rows(), rows(), **weighed) == ESIZE


def test_so_many_query_heads_of_a_kv_head_are_refused():
    size = spqt.lib().spqt_kv_workspace_bytes
    out = ctypes.c_size_t()
    assert size(1, 1, 1 << 20, 1, 64, 1, ctypes.byref(out)) == 0 and size(1, 1, 4 << 20, 4, 64, 1, ctypes.byref(out)) == 0
    assert size(1, 1, (1 << 20) + 1, 1, 64, 1, ctypes.byref(out)) == ESHAPE
    assert attention(cache(kv_heads=1, weights=1 << 20), rows(), rows(data=1 << 21), lse=1 << 22, heads=1 << 23, size=16) == ESHAPE


def test_places_by_the_inverse():
    """The rule of kv_weigh.hip in fp32, at and beside every whole position: 32 rows from any of a kv head's query heads on."""
    f = lambda x: torch.tensor(x, dtype=torch.float32)  # noqa: E731
    for group in (1, 2, 3, 5, 7, 8, 40, 641, 4095, 65537, (1 << 20) - 1, 1 << 20):
        inverse = f(1.0) / f(float(group))
        n = torch.cat([torch.arange(min(group + 32, 4096)), torch.arange(max(0, group - 64), group + 32), torch.arange(32) + group - 1])
        n = n[n < group + 31]
        assert torch.equal(((n.float() + f(0.5)) * inverse).long(), n // group)
