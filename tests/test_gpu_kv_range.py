"""The key/value cache over its whole range: how many bits probabilities have, whichever kernel a call takes, and what lies far from 1.

Attention's tolerance, per output, with u = 2^-11 (fp16) or 2^-8 (bf16), e = 2^-24 and the oracle's sums sway = scale sum |q| |k| and
spread = sum p |v|: a score is off by at most d = (D + 8) e sway, a probability by 2 d + (L + 64) e of itself and by 2^-21, since it is held in
two fp16 numbers (2^-11 of 2^-11 of itself at most, and as much again for the numbers that it is made of); but no less than fp16's smallest step
leaves: half of 2^-24 in units of 2^-15 of the largest term of the ROW, the product of a probability and its block's value scale, of which the units
may be four times (whole powers of two of either).  Many rows: of the largest probability times the largest scale that the row sees, though no more
than 2^14 of the former.  The output: u |out| + spread times that + L e spread + L 2^-40 times 127 of that unit, and half of the type's smallest number."""
import pytest
import torch

import oracle as gemv_oracle
from oracle import kv as oracle
from test_gpu_kv import CASES, Cache, E, EITHER, MANY, attend, case_cache, gpu, widen  # noqa: F401

from workloads import make_weights, make_x, quantile_threshold

pytestmark = pytest.mark.gpu

# above 16 rows of a kv head, in sixteens
SIXTEENS = [
    (8, 1, 128, "float16", [700], None, 4, 0),
    (16, 1, 256, "bfloat16", [300, 90], None, 4, 50),
    (6, 2, 64, "float16", [400, 31], [20, 2], 20, 0),
]


def largest_terms(c, q, each, window, scale):
    """For every row and query head: the largest product of a probability and its block's value scale, and of any probability and any such scale."""
    S, n, Hq, dim = q.shape
    H = c.codes.shape[1]
    codes, scales, q = c.codes.cpu(), c.scales.cpu().double(), q.cpu().double()
    found = torch.zeros((2, S, n, Hq), dtype=torch.float64)
    for s in range(S):
        L = c.length_of[s]
        for h in range(H):
            k = oracle.token_values(codes, scales, c.table_host[s], h, 0, L)
            of = scales[c.table_host[s].long(), h, 1].repeat_interleave(64)[:L]
            for i in range(each[s]):
                at = L - each[s] + i
                low = max(0, at - window + 1) if window > 0 else 0
                if at < 0:
                    continue
                for j in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    p = torch.softmax((k[low : at + 1] @ q[s, i, j]) * scale, 0)
                    found[0, s, i, j] = (p * of[low : at + 1]).max()
                    found[1, s, i, j] = p.max() * of[low : at + 1].max()
    return found


def within(c, q, counts, window, out, scale=None, held=2.0 ** -21):
    """The largest error, in units of what is allowed."""
    seqs, rows, heads, dim = q.shape
    each = [rows] * seqs if counts is None else counts
    scale = dim ** -0.5 if scale is None else scale
    want, _, _, sway, spread, _ = oracle.attention(c.codes.cpu(), c.scales.cpu(), c.table_host, c.length_of, q.cpu(), each, scale, window)
    want = want.clamp(-torch.finfo(q.dtype).max, torch.finfo(q.dtype).max)      # outputs are the type's numbers, as values read back are
    L = max(c.length_of)
    u, smallest = (2.0 ** -11, 2.0 ** -24) if q.dtype == torch.float16 else (2.0 ** -8, 2.0 ** -133)
    off = 2 * (dim + 8) * E * sway + (L + 64) * E + held
    term, separate = largest_terms(c, q, each, window, scale)
    many = rows * heads // c.kv_heads > 64               # (those that the kernel for a few rows takes all the same are no further off)
    floor = L * 2.0 ** -38 * 127 * (torch.minimum(separate, term * 2.0 ** 14) if many else term)
    bound = u * want.abs() + (spread * (off[..., None] + L * E) + floor[..., None]) * (1 + u) + smallest / 2
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
    c = steep_cache(gpu, dtype, sizes, kv_heads, dim, len(sizes) + dim)
    q = (0.05 * torch.randn((1, rows, heads, dim), generator=c.gen)).to(c.dtype).cuda()
    if wide:
        widen(c)
    out, lse = attend(gpu, c, q, None)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert within(c, q, None, 0, out) <= 1.0


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("size", [1e6, 1e12, 1e30])
@pytest.mark.parametrize("rows", [4, 65])
def test_large_values_that_other_rows_see(gpu, rows, size, dim):  # noqa: F811
    """The first row sees one token of the block of large values, the rows beside it none; every wavefront has several blocks."""
    c = steep_cache(gpu, "bfloat16", [size] + [1.0] * 15, 2, dim, 7 + dim)
    window = 1024 - rows - 63 + 1
    q = (0.05 * torch.randn((1, rows, 8, dim), generator=c.gen)).bfloat16().cuda()
    for wide in (False, True):
        if wide:
            widen(c)
        out, _ = attend(gpu, c, q, None, window)
        assert float(out[:, 0].min()) > size * 1e-4 and float(out[:, 1:].max()) < 2.0 and float(out[:, 1:].min()) > 0.5
        assert within(c, q, None, window, out) <= 1.0


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("place", [0, 1])
@pytest.mark.parametrize("heads,kv_heads,rows,wide", FORMS)
def test_large_values_that_get_no_weight(gpu, heads, kv_heads, rows, wide, place, dim):  # noqa: F811
    """A block of large values whose keys point away from every query, before and after the others: probabilities of 2^-140 and less."""
    sizes = [1.0] * 16
    sizes[place] = 1e20
    c = Cache(gpu, 1, kv_heads, dim, torch.bfloat16, 16, 11 + dim)
    x = torch.randn((1, 1024, 2 * kv_heads, dim), generator=c.gen)
    each = torch.tensor(sizes).repeat_interleave(64)[None, :, None, None]
    x[:, :, kv_heads:] = each * (0.9 + 0.01 * x[:, :, kv_heads:])
    x[:, :, :kv_heads] = torch.where(each > 1, -10.0, 0.1) + 0.1 * x[:, :, :kv_heads]
    c.append(1024, x=x.bfloat16())
    q = (1.5 + 0.01 * torch.randn((1, rows, heads, dim), generator=c.gen)).bfloat16().cuda()
    if wide:
        widen(c)
    out, _ = attend(gpu, c, q, None)
    assert float(out.max()) < 2.0 and float(out.min()) > 0.5
    assert within(c, q, None, 0, out) <= 1.0


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("heads,kv_heads,rows,wide", FORMS)
@pytest.mark.parametrize("blocks", [1, 30, 100])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_the_largest_values_there_are(gpu, dtype, blocks, heads, kv_heads, rows, wide, dim):  # noqa: F811
    """Sums over up to 6400 tokens that meet in shared memory and in the workspace; 127 scale is beyond the type's largest number."""
    c = Cache(gpu, 1, kv_heads, dim, getattr(torch, dtype), blocks, 13 + dim)
    x = torch.randn((1, 64 * blocks, 2 * kv_heads, dim), generator=c.gen)
    signs = torch.where(torch.arange(dim) % 3 == 0, -1.0, 1.0)
    x[:, :, kv_heads:] = torch.finfo(c.dtype).max * signs
    c.append(64 * blocks, x=x.to(c.dtype))
    q = (0.05 * torch.randn((1, rows, heads, dim), generator=c.gen)).to(c.dtype).cuda()
    if wide:
        widen(c)
    out, _ = attend(gpu, c, q, None)                       # (6 of 70 rows lie before the first of 64 tokens)
    assert bool(torch.isfinite(out).all())
    assert within(c, q, None, 0, out) <= 1.0


@pytest.mark.parametrize("case", [(64, 8, 128, "float16", [1500], None, 1, 0), (8, 1, 128, "float16", [2100], None, 70, 0)], ids=["few", "many"])
def test_a_gemv_does_not_take_words_of_an_attention_for_its_own(gpu, case):  # noqa: F811
    """On an attention's workspace it gives NaN until the workspace is prepared again; with its own it is right."""
    _, spqt = gpu
    M, K = 1024, 2048
    w, x_np = make_weights(M, K, 77), make_x(K, "laplace", 78)
    thr = quantile_threshold(x_np, 0.5)
    want = torch.from_numpy(gemv_oracle.gemv(w["q_rowmajor"], w["scales"], x_np, thr)[0])
    packed, x = torch.from_numpy(spqt.spqt_pack(w["q_rowmajor"], w["scales"])).cuda(), torch.from_numpy(x_np[0].copy()).cuda()
    idx, count = torch.empty(K, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    spqt.spqt_gather(x, thr, idx, count)
    y = torch.zeros(M, device="cuda")
    c, q = case_cache(gpu, case, 36)
    expected, _ = attend(gpu, c, q, None)
    size = max(spqt.spqt_workspace_bytes(M, K, 1), spqt.spqt_kv_workspace_bytes(1, case[6], case[0], case[1], case[2], 64))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def gemv():
        spqt.spqt_gemv(packed, M, K, x, idx, count, y, ws, splits=4, waves=4)
        return bool(((y.cpu().double() - want).abs() <= 1e-2 + 2e-3 * want.abs()).all())

    spqt.spqt_workspace_init(ws)
    assert gemv() and gemv()
    out, _ = attend(gpu, c, q, None, workspace=ws)         # (a GEMV leaves the workspace all zeros)
    assert out.equal(expected)
    gemv()
    assert bool(y.isnan().all())
    spqt.spqt_workspace_init(ws)
    assert gemv()


@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("size", [1 << 31, (1 << 32) + 16, -(1 << 32) + 16, 1 << 64, float("inf"), "many"])
def test_numbers_beyond_32_bits_are_refused(gpu, size, fast, monkeypatch):  # noqa: F811
    """Not taken by their lowest 32 bits: a window of 2^32 + 16 would be one of 16."""
    _, spqt = gpu
    if not fast:
        from paper_2511_04477_amd import binding
        monkeypatch.setattr(binding, "_fast", None)
    c, q = case_cache(gpu, CASES[2], 37)
    out, ws = torch.zeros_like(q), spqt.new_kv_workspace(3, 1, 8, 2, 128, 4)
    with pytest.raises(spqt.SpqtError):
        spqt.spqt_kv_attention(c.codes, c.scales, c.table, c.lengths, q, out, ws, window=size)
    new_lengths = torch.zeros(3, dtype=torch.int32, device="cuda")
    for keep, recent in ((64, size), (size, 3)):
        kept = torch.zeros((3, 2, 64), dtype=torch.int32, device="cuda")
        with pytest.raises(spqt.SpqtError):
            spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, c.table[:, :2].contiguous(), c.lengths, keep, recent, c.table[:, 2:].contiguous(), new_lengths, kept)
    assert not bool(out.any()) and not bool(new_lengths.any())
    for at in range(6):
        sizes = [3, 1, 8, 2, 128, 4]
        sizes[at] = size
        with pytest.raises(spqt.SpqtError):
            spqt.spqt_kv_workspace_bytes(*sizes)


def test_windows_up_to_31_bits_see_everything(gpu):  # noqa: F811
    c, q = case_cache(gpu, CASES[2], 37)
    want = attend(gpu, c, q, None)
    for window in (1 << 24, (1 << 31) - 1):
        got = attend(gpu, c, q, None, window)
        assert got[0].equal(want[0]) and got[1].equal(want[1])


@pytest.mark.parametrize("case", [CASES[i] for i in (2, 7, 8, 12, 14)] + MANY[:2], ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_outputs_over_the_queries(gpu, case):  # noqa: F811
    """Without weights the same as elsewhere; with weights, whose queries are read after the outputs are written, refused."""
    _, spqt = gpu
    c, q = case_cache(gpu, case, 38)
    counts = None if case[5] is None else torch.tensor(case[5], dtype=torch.int32, device="cuda")
    want, want_lse = attend(gpu, c, q, case[5], case[7])
    ws = spqt.new_kv_workspace(len(case[4]), case[6], case[0], case[1], case[2], c.max_blocks)
    lse, weights = torch.zeros_like(want_lse), c.weights.clone()
    before = q.clone()
    with pytest.raises(spqt.SpqtError):
        spqt.spqt_kv_attention(c.codes, c.scales, c.table, c.lengths, q, q, ws, counts=counts, window=case[7], lse=lse, weights=c.weights)
    assert q.equal(before) and c.weights.equal(weights)
    spqt.spqt_kv_attention(c.codes, c.scales, c.table, c.lengths, q, q, ws, counts=counts, window=case[7], lse=lse)
    assert q.equal(want) and lse.equal(want_lse)
