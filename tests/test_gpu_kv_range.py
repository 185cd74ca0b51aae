"""The key/value cache over its whole range: how many bits probabilities have, whichever kernel a call takes, and what lies far from 1.

Attention's tolerance, per output, with u = 2^-11 (fp16) or 2^-8 (bf16), e = 2^-24 and the oracle's sums sway = scale sum |q| |k| and
spread = sum p |v|: a score is off by at most d = (D + 8) e sway, a probability by 2 d + (L + 64) e of itself and by 2^-21, since it is held in
two fp16 numbers (2^-11 of 2^-11 of itself at most, and as much again for the numbers that it is made of); but no less than fp16's smallest step
leaves: half of 2^-24 in units of 2^-15 of the largest value scale there is.  The output: u |out| + spread times that + L e spread + L 2^-40 times
127 of that scale, and half of the type's smallest number."""
import pytest

from oracle import kv as oracle
from test_gpu_kv import E, EITHER, MANY, attend, case_cache, gpu, widen  # noqa: F401

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
