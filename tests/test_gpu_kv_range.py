"""The key/value cache over its whole range: how many bits probabilities have, whichever kernel a call takes, and what lies far from 1.

Attention's tolerance, per output, with u = 2^-11 (fp16) or 2^-8 (bf16), e = 2^-24 and the oracle's sums sway = scale sum |q| |k| and
spread = sum p |v|: a score is off by at most d = (D + 8) e sway, a probability by 2 d + (L + 64) e of itself and by 2^-21, since it is held in
two fp16 numbers (2^-11 of 2^-11 of itself at most, and as much again for the numbers that it is made of); but no less than fp16's smallest step
leaves: half of 2^-24 in units of 2^-15 of the largest value scale there is.  The output: u |out| + spread times that + L e spread + L 2^-40 times
127 of that scale, and half of the type's smallest number."""
import pytest

from oracle import kv as oracle
from test_gpu_kv import Cache, E, EITHER, MANY, attend, case_cache, gpu, widen  # noqa: F401

pytestmark = pytest.mark.gpu

# above 16 rows of a kv head, in sixteens
SIXTEENS = [
    (8, 1, 128, "float16", [700], None, 4, 0),
    (16, 1, 256, "bfloat16", [300, 90], None, 4, 50),
    (6, 2, 64, "float16", [400, 31], [20, 2], 20, 0),
]


def within(c, q, counts, window, out, scale=None, held=2.0 ** -21):
    torch = c.torch
    seqs, rows, heads, dim = q.shape
    each = [rows] * seqs if counts is None else counts
    scale = dim ** -0.5 if scale is None else scale
    want, _, _, sway, spread, _ = oracle.attention(c.codes.cpu(), c.scales.cpu(), c.table_host, c.length_of, q.cpu(), each, scale, window)
    L = max(c.length_of)
    u, smallest = (2.0 ** -11, 2.0 ** -24) if q.dtype == torch.float16 else (2.0 ** -8, 2.0 ** -133)
    off = 2 * (dim + 8) * E * sway + (L + 64) * E + held
    floor = L * 2.0 ** -40 * 127 * float(c.scales[c.table[:, : -(-L // 64)].long()][..., 1].max())
    bound = u * want.abs() + (spread * (off[..., None] + L * E) + floor) * (1 + u) + smallest / 2
    return float(((out.cpu().double() - want).abs() / bound).max())


@pytest.mark.parametrize("case,wide", [(c, False) for c in SIXTEENS + MANY] + [(c, w) for c in EITHER for w in (False, True)],
                         ids=lambda c: "-".join(str(x) for x in c).replace(" ", "") if isinstance(c, tuple) else None)
def test_probabilities_have_twenty_two_bits_in_every_kernel(gpu, case, wide):  # noqa: F811
    c, q = case_cache(gpu, case, 35)
    if wide:
        widen(c)
    out, _ = attend(gpu, c, q, case[5], case[7])
    assert within(c, q, case[5], case[7], out) <= 1.0


# sizes of the values, a block each: a block of zeros has the scale 2^-100
STEEP = [
    ("float16", [8.0] * 40 + [0.0]),
    ("float16", [1.0] * 140 + [0.0] + [1.0] * 4),
    ("bfloat16", [1000.0, 0.0]),
    ("float16", [1000.0] * 10 + [0.0] + [1000.0] * 2),     # one part, with many rows
    ("float16", [100.0] * 46 + [0.0] + [100.0] * 17),      # several parts: the block of zeros is the seventh of its part
    ("bfloat16", [1e30, 1e-30, 1.0, 1e20, 0.0, 1e-10, 1e12] * 2),
    ("float16", [0.0, 6e-8, 0.0, 1e-4, 60000.0, 0.0]),
]
# query heads, kv heads, rows, wide tables: a few rows, some that are a few or many by the tables' room, many rows
FORMS = [(8, 2, 1, False), (8, 1, 12, False), (8, 1, 12, True), (8, 1, 70, False)]


def steep_cache(gpu, dtype, sizes, kv_heads, dim, seed):  # noqa: F811
    torch, _ = gpu
    c = Cache(gpu, 1, kv_heads, dim, getattr(torch, dtype), len(sizes), seed)
    x = torch.randn((1, 64 * len(sizes), 2 * kv_heads, dim), generator=c.gen)
    each = torch.tensor(sizes, dtype=torch.float64).float().repeat_interleave(64)[None, :, None, None]
    x[:, :, kv_heads:] = each * (0.9 + 0.01 * x[:, :, kv_heads:])          # values of one sign and about one size
    c.append(64 * len(sizes), x=x.to(c.dtype))
    return c


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("heads,kv_heads,rows,wide", FORMS)
@pytest.mark.parametrize("dtype,sizes", STEEP, ids=lambda x: x if isinstance(x, str) else f"{len(x)}x{x[0]}")
def test_blocks_of_zeros_and_of_very_different_values(gpu, dtype, sizes, heads, kv_heads, rows, wide, dim):  # noqa: F811
    """Rows that weigh all tokens about the same."""
    torch, _ = gpu
    c = steep_cache(gpu, dtype, sizes, kv_heads, dim, len(sizes) + dim)
    q = (0.05 * torch.randn((1, rows, heads, dim), generator=c.gen)).to(c.dtype).cuda()
    if wide:
        widen(c)
    out, lse = attend(gpu, c, q, None)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert within(c, q, None, 0, out) <= 1.0
