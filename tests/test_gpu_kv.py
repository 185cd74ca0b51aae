"""The key/value cache in 8 bits on the GPU against the 64-bit oracle (oracle/kv.py).

What is quantized is exact: codes, scales, tails and values read back are compared bit for bit, and so is everything that a call has
to leave alone.  Attention's tolerance, per output, with u = 2^-11 (fp16) or 2^-8 (bf16), e = 2^-24 and the oracle's sums
sway = scale sum |q| |k| and spread = sum p |v| :
    a score is off by at most d = (D + 8) e sway (sums of D products in fp32), a probability by 2 d + (L + 64) e of itself (its own
    score and the sum of L), and by another 2^-21 where it is held in two fp16 numbers (up to 16 rows a kv head) or 2^-11 where in one,
    but no less than fp16's smallest step leaves: times 2^15 and the block's scale over the largest one, half of 2^-24;
    out: u |out| + spread times that + L e spread + L 2^-40 times 127 of the largest scale, and half of the type's smallest number;
    lse: 2 d + (L + 64) e + 4 e |lse|;  weights: the sum over the rows of what their probabilities are off by, 4 e |lse| more for the use of lse."""
import math

import pytest

from oracle import kv as oracle

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2511_04477_amd as spqt
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spqt.lib()
    return torch, spqt


class Cache:
    """A pool with more pages than are used, in random order, and a mirror of what it has to hold."""

    def __init__(self, gpu, seqs, kv_heads, dim, dtype, max_blocks, seed, weights=True):
        self.torch, self.spqt = torch, spqt = gpu
        self.gen = torch.Generator().manual_seed(seed)
        self.seqs, self.kv_heads, self.dim, self.dtype, self.max_blocks = seqs, kv_heads, dim, dtype, max_blocks
        self.pages = seqs * max_blocks + 2
        self.codes, self.scales, self.tail, self.weights = spqt.new_kv_cache(self.pages, kv_heads, dim, seqs, dtype, weights)
        self.codes.copy_(torch.randint(0, 256, self.codes.shape, generator=self.gen, dtype=torch.uint8))
        self.scales.copy_(torch.randn(self.scales.shape, generator=self.gen))
        self.tail.fill_(7.0)
        if weights:
            self.weights.copy_(torch.rand(self.weights.shape, generator=self.gen))
        order = torch.randperm(self.pages, generator=self.gen)
        self.table_host = order[: seqs * max_blocks].view(seqs, max_blocks).to(torch.int32)
        self.table = self.table_host.cuda()
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.length_of = [0] * seqs
        self.tokens = [[torch.zeros((0, kv_heads, dim), dtype=dtype) for _ in range(seqs)] for _ in range(2)]

    def values(self, rows, spread=1.0):
        torch = self.torch
        x = torch.randn((self.seqs, rows, 2 * self.kv_heads, self.dim), generator=self.gen)
        x *= torch.exp(spread * torch.randn((self.seqs, rows, 1, 1), generator=self.gen))
        return x.to(self.dtype)

    def append(self, rows, counts=None, x=None, **more):
        """counts: tokens of every sequence, None for all rows; keys and values are slices of one tensor."""
        torch = self.torch
        x = self.values(rows) if x is None else x
        each = [rows] * self.seqs if counts is None else counts
        for s, n in enumerate(each):
            self.length_of[s] += n
            for which in (0, 1):
                part = x[s, :n, which * self.kv_heads : (which + 1) * self.kv_heads]
                self.tokens[which][s] = torch.cat([self.tokens[which][s], part])
        self.lengths.copy_(torch.tensor(self.length_of, dtype=torch.int32))
        k, v = x.cuda().split([self.kv_heads, self.kv_heads], dim=2)
        c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        self.spqt.spqt_kv_append(self.codes, self.scales, self.tail, self.table, self.lengths, k, v, counts=c, weights=self.weights, **more)

    def check(self, before, new):
        """The pool against the oracle, and against its state before the last call where nothing was appended. new: tokens of that call per sequence."""
        torch = self.torch
        codes, scales, tail = self.codes.cpu(), self.scales.cpu(), self.tail.cpu()
        codes_before, scales_before, tail_before, weights_before = before
        expected_scales = scales_before.clone()
        expected_tail = tail_before.clone()
        expected_weights = None if weights_before is None else weights_before.clone()
        same = torch.ones(codes.shape, dtype=torch.bool)         # where the pool must be as before
        for s in range(self.seqs):
            n = self.length_of[s]
            if new[s] == 0:
                continue
            for b in range((n - new[s]) // 64, (n - 1) // 64 + 1):
                page, here = int(self.table_host[s, b]), min(64, n - 64 * b)
                first = max(0, n - new[s] - 64 * b)
                if expected_weights is not None:
                    expected_weights[page, :, first:here] = 0.0
                for h in range(self.kv_heads):
                    for which in (0, 1):
                        x = self.tokens[which][s][64 * b : 64 * b + here, h].double()
                        want, scale = oracle.quantize(x)
                        expected_scales[page, h, which] = scale
                        if want is None:
                            want = torch.zeros(x.shape, dtype=torch.long) - 127
                            got = oracle.page_codes(codes[page, h], which)[first:here]
                            assert bool(((got >= -127) & (got <= 127)).all())
                        else:
                            assert torch.equal(oracle.page_codes(codes[page, h], which)[:here], want), (s, b, h, which)
                        if which == 0:
                            same[page, h, 0, :here] = False
                        else:
                            same[page, h, 1].view(self.dim, 64)[:, oracle.PLACE[:here]] = False
                        if b == (n - 1) // 64 and here < 64:
                            expected_tail[s, h, which, first:here] = self.tokens[which][s][64 * b + first : n, h]
        assert torch.equal(scales.view(torch.int32).masked_fill(scales.isnan(), 0), expected_scales.view(torch.int32).masked_fill(expected_scales.isnan(), 0))
        assert torch.equal(scales.isnan(), expected_scales.isnan())
        assert torch.equal(codes[same], codes_before[same])
        assert torch.equal(tail.view(torch.int16), expected_tail.view(torch.int16))
        if expected_weights is not None:
            assert torch.equal(self.weights.cpu(), expected_weights)

    def state(self):
        return self.codes.cpu(), self.scales.cpu(), self.tail.cpu(), None if self.weights is None else self.weights.cpu()


HEADS = [(1, 64), (3, 128), (2, 192), (1, 256)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("kv_heads,dim", HEADS)
@pytest.mark.parametrize("pieces", [[1], [64], [63, 1, 1], [5, 59, 64, 3], [130, 7, 200], [1, 2, 3, 1, 1, 60]])
def test_append_in_pieces(gpu, dtype, kv_heads, dim, pieces):
    torch, _ = gpu
    c = Cache(gpu, 2, kv_heads, dim, getattr(torch, dtype), 6, sum(pieces) + dim)
    for n in pieces:
        before = c.state()
        c.append(n)
        c.check(before, [n, n])


def test_append_of_uneven_counts(gpu):
    torch, _ = gpu
    c = Cache(gpu, 5, 2, 128, torch.float16, 5, 3)
    for counts in ([70, 0, 1, 33, 64], [0, 5, 70, 31, 1], [1, 0, 0, 0, 0], [2, 59, 68, 65, 63]):
        before = c.state()
        c.append(70, counts)
        c.check(before, counts)


def test_what_a_block_holds_does_not_depend_on_the_calls(gpu):
    torch, _ = gpu
    whole, single = (Cache(gpu, 1, 2, 128, torch.float16, 2, 9) for _ in range(2))
    x = whole.values(100, 2.0)
    whole.append(100, x=x)
    for t in range(100):
        single.append(1, x=x[:, t : t + 1])
    for b, n in ((0, 64), (1, 36)):
        page = int(whole.table_host[0, b])
        assert torch.equal(whole.scales[page], single.scales[page])
        for h in range(2):
            for which in (0, 1):
                assert torch.equal(oracle.page_codes(whole.codes[page, h].cpu(), which)[:n], oracle.page_codes(single.codes[page, h].cpu(), which)[:n])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_append_of_extreme_values(gpu, dtype):
    torch, _ = gpu
    dtype = getattr(torch, dtype)
    largest, tiny = torch.finfo(dtype).max, 6e-8 if dtype == torch.float16 else 1e-40
    c = Cache(gpu, 1, 1, 64, dtype, 4, 5)
    for fill in (0.0, tiny, -tiny, 1.0, largest, -largest):
        before = c.state()
        x = c.values(40) * 0 + fill
        x[0, 3, :, 5] = 0.0
        c.append(40, x=x.to(dtype))
        c.check(before, [40])
    assert bool(torch.isfinite(c.scales[c.table_host[0].long().cuda()]).all())


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_append_of_what_is_not_a_number(gpu, bad):
    torch, _ = gpu
    c = Cache(gpu, 1, 2, 128, torch.float16, 4, 6)
    c.append(70)
    x = c.values(3)
    x[0, 1, 2, 7] = bad                            # a value of head 0
    before = c.state()
    c.append(3, x=x)
    c.check(before, [3])
    before = c.state()
    c.append(61)                                   # the block stays what it is, the next one is sound
    c.check(before, [61])
    nan = c.scales.isnan().nonzero().tolist()
    assert nan == [[int(c.table_host[0, 1]), 0, 1]]


def test_append_leaves_alone_what_has_no_page(gpu):
    torch, spqt = gpu
    c = Cache(gpu, 2, 1, 64, torch.float16, 2, 8)
    c.table[0, 1] = c.pages
    c.table[1, 0] = -1
    before = c.state()
    x = c.values(100).cuda()
    c.lengths.copy_(torch.tensor([100, 1000], dtype=torch.int32))          # the second is taken as 128: its first 28 tokens are at 28 .. 55
    spqt.spqt_kv_append(c.codes, c.scales, c.tail, c.table, c.lengths, x[:, :, :1], x[:, :, 1:], weights=c.weights)
    touched = {int(c.table_host[0, 0]), int(c.table_host[1, 1])}
    after = c.state()
    for page in range(c.pages):
        assert (page in touched) != torch.equal(after[1][page], before[1][page])
        if page not in touched:
            assert torch.equal(after[0][page], before[0][page])
    c.lengths.copy_(torch.tensor([-5, 30], dtype=torch.int32))             # nothing; and 70 of the 100 rows lie before the first token
    before = c.state()
    spqt.spqt_kv_append(c.codes, c.scales, c.tail, c.table, c.lengths, x[:, :, :1], x[:, :, 1:], counts=torch.tensor([3, 200], dtype=torch.int32, device="cuda"))
    after = c.state()
    assert torch.equal(before[0], after[0])                                # (block 0 of sequence 1 has no page)
    assert torch.equal(after[2][0].view(torch.int16), before[2][0].view(torch.int16))
    assert torch.equal(after[2][1, 0, 0, :30], x[1, 70:100, 0].cpu())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("kv_heads,dim", HEADS)
def test_read(gpu, dtype, kv_heads, dim):
    torch, spqt = gpu
    dtype = getattr(torch, dtype)
    c = Cache(gpu, 3, kv_heads, dim, dtype, 4, 12 + dim)
    c.append(200, [200, 63, 0])
    x = torch.tensor([torch.finfo(dtype).max]).to(dtype).expand(3, 1, 2 * kv_heads, dim).clone()
    c.append(1, [1, 0, 0], x=x)                     # the largest number there is: 127 scale rounds beyond it
    for rows, counts in ((300, [201, 63, 0]), (7, [5, 7, 7]), (130, [129, 100, 1]), (1, None)):
        outs = [torch.full((3, rows, kv_heads, dim + 8), 3.0, dtype=dtype, device="cuda") for _ in range(2)]
        k, v = (o[..., :dim] for o in outs)
        spqt.spqt_kv_read(c.codes, c.scales, c.table, c.lengths, k, v, counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
        codes, scales = c.codes.cpu(), c.scales.cpu()
        for which, got in ((0, k), (1, v)):
            assert bool((outs[which][..., dim:] == 3.0).all())
            for s in range(3):
                L, n = c.length_of[s], rows if counts is None else counts[s]
                for h in range(kv_heads):
                    held = oracle.rounded(oracle.token_values(codes, scales, c.table_host[s], h, which, L), dtype)
                    want = torch.zeros((rows, dim), dtype=dtype)
                    for i in range(n):
                        if L - n + i >= 0:
                            want[i] = held[L - n + i]
                    assert torch.equal(got[s, :, h].cpu().view(torch.int16), want.view(torch.int16)), (which, s, h)


def attend(gpu, c, q, counts, window=0, scale=None, weigh=False, decay=1.0, stream=None, workspace=None, lse=True):
    torch, spqt = gpu
    seqs, rows, heads, dim = q.shape
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
    lse = torch.full((seqs, rows, heads), 9.0, device="cuda") if lse else None
    ws = spqt.new_kv_workspace(seqs, rows, heads, c.kv_heads, dim, c.table.shape[1]) if workspace is None else workspace
    spqt.spqt_kv_attention(c.codes, c.scales, c.table, c.lengths, q, out, ws, scale=scale, counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"),
                           window=window, lse=lse, weights=c.weights if weigh else None, decay=decay, stream=stream)
    return out, lse


def compare(gpu, c, q, counts, window, out, lse, scale=None, weights=None, before=None, decay=1.0):
    torch, _ = gpu
    seqs, rows, heads, dim = q.shape
    each = [rows] * seqs if counts is None else counts
    scale = dim ** -0.5 if scale is None else scale
    want, want_lse, sums, sway, spread, weight_sway = oracle.attention(c.codes.cpu(), c.scales.cpu(), c.table_host, c.length_of, q.cpu(), each, scale, window)
    L = max(c.length_of)
    u = 2.0 ** -11 if q.dtype == torch.float16 else 2.0 ** -8
    smallest = 2.0 ** -24 if q.dtype == torch.float16 else 2.0 ** -133
    d = (dim + 8) * E * sway
    held = 2.0 ** -21 if rows * heads // c.kv_heads <= 16 else 2.0 ** -11
    off = 2 * d + (L + 64) * E + held
    floor = L * 2.0 ** -40 * 127 * float(c.scales[c.table[:, : -(-L // 64)].long()][..., 1].nan_to_num(0.0).max())
    bound = u * want.abs() + (spread * (off[..., None] + L * E) + floor) * (1 + u) + smallest / 2
    got = out.cpu().double()
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    empty = want_lse == -math.inf
    got = lse.cpu().double()
    assert torch.equal(got == -math.inf, empty)
    limit = 2 * d + (L + 64) * E + 4 * E * want_lse.abs()
    assert bool(((got - want_lse).abs() <= limit)[~empty].all())
    assert bool((out.cpu()[empty] == 0).all())
    if weights is None:
        return
    most = float(want_lse[~empty].abs().max()) if bool((~empty).any()) else 0.0
    got, expected, limits = weights.cpu(), before.clone().double(), torch.zeros(before.shape, dtype=torch.float64)
    for s in range(seqs):
        for b in range(-(-c.length_of[s] // 64)):
            page, n = int(c.table_host[s, b]), min(64, c.length_of[s] - 64 * b)
            for h in range(c.kv_heads):
                part = slice(64 * b, 64 * b + n)
                w = sums[s][h][part]
                expected[page, h, :n] = w + (decay * expected[page, h, :n] if decay else 0.0)
                limits[page, h, :n] = (4 * (dim + 8) * E * weight_sway[s][h][part] + w * ((L + 64 + rows * heads) * E + 4 * E * most + 2.0 ** -20)
                                       + 4 * E * expected[page, h, :n].abs() + 2.0 ** -126)
    assert bool(((got.double() - expected).abs() <= limits).all()), float(((got.double() - expected).abs() - limits).max())


CASES = [
    # heads, kv heads, dim, type, lengths, counts (None: `rows` of each), rows, window
    (1, 1, 64, "float16", [1], None, 1, 0),
    (8, 8, 128, "float16", [64, 65, 63], None, 1, 0),
    (8, 2, 128, "bfloat16", [200, 1, 129], None, 1, 0),
    (12, 4, 64, "float16", [333, 0, 17, 64], [1, 0, 1, 1], 1, 0),
    (16, 1, 256, "bfloat16", [700, 300], None, 1, 0),
    (5, 1, 192, "float16", [130, 7], None, 3, 0),
    (40, 40, 64, "bfloat16", [90], None, 4, 20),
    (64, 8, 128, "float16", [1500], None, 1, 0),
    (64, 8, 128, "bfloat16", [2100, 40], None, 2, 100),
    (8, 2, 128, "float16", [70, 300, 64], [5, 1, 3], 5, 0),
    (32, 8, 128, "float16", [11, 100], [11, 9], 11, 3),
    (4, 4, 128, "bfloat16", [257], None, 17, 0),
    (6, 2, 64, "float16", [400, 31], [40, 31], 40, 0),
    (8, 1, 128, "float16", [150, 640], [150, 70], 150, 0),
    (4, 2, 256, "bfloat16", [300], None, 300, 50),
    (2, 1, 192, "float16", [513, 0, 190], [200, 0, 190], 200, 0),
    (3, 3, 128, "bfloat16", [5, 700], [5, 1], 30, 1),
    (8, 2, 64, "float16", [40], None, 60, 0),          # rows before the first token see nothing
    (8, 1, 128, "float16", [2100], None, 40, 0),       # many rows, tokens in parts
    (4, 2, 64, "bfloat16", [1500, 30, 0, 800], [50, 30, 0, 1], 50, 300),
    (6, 1, 192, "bfloat16", [1100, 1030], [33, 20], 33, 0),
    (4, 1, 256, "float16", [1300], None, 70, 0),
]


def case_cache(gpu, case, seed):
    torch, _ = gpu
    heads, kv_heads, dim, dtype, lengths, counts, rows, window = case
    dtype = getattr(torch, dtype)
    c = Cache(gpu, len(lengths), kv_heads, dim, dtype, max(1, -(-max(lengths) // 64)), seed)
    c.append(max(1, max(lengths)), lengths)
    q = torch.randn((len(lengths), rows, heads + 2, dim), generator=c.gen) * torch.exp(torch.randn((1, 1, heads + 2, dim), generator=c.gen))
    return c, q.to(dtype).cuda()[:, :, 1:-1]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_attention(gpu, case):
    heads, kv_heads, dim, dtype, lengths, counts, rows, window = case
    c, q = case_cache(gpu, case, 31)
    before = c.state()
    out, lse = attend(gpu, c, q, counts, window)
    compare(gpu, c, q, counts, window, out, lse)
    for a, b in zip(before, c.state()):
        assert a.equal(b)                              # the cache is read only
    again, lse_again = attend(gpu, c, q, counts, window)
    assert out.equal(again) and lse.equal(lse_again)   # sums are joined in a fixed order
    without, _ = attend(gpu, c, q, counts, window, lse=False)
    assert out.equal(without)


@pytest.mark.parametrize("decay", [1.0, 0.0, 0.75])
@pytest.mark.parametrize("case", [CASES[i] for i in (0, 2, 3, 7, 9, 12, 13, 15, 17)], ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_attention_with_weights(gpu, case, decay):
    torch, _ = gpu
    heads, kv_heads, dim, dtype, lengths, counts, rows, window = case
    c, q = case_cache(gpu, case, 32)
    c.weights.copy_(torch.rand(c.weights.shape, generator=c.gen))
    if decay == 0.0:
        c.weights.view(-1)[::3] = math.nan              # what is not read
    before = c.weights.cpu()
    out, lse = attend(gpu, c, q, counts, window, weigh=True, decay=decay)
    if decay == 0.0:
        for s, n in enumerate(c.length_of):
            inside = torch.arange(c.max_blocks * 64) < n
            assert not bool(c.weights.cpu()[c.table_host[s].long()].transpose(1, 2).flatten(0, 1)[inside].isnan().any())
        before, c.weights = before.nan_to_num(0.0), c.weights.nan_to_num(0.0)
    compare(gpu, c, q, counts, window, out, lse, weights=c.weights, before=before, decay=decay)


@pytest.mark.parametrize("rows", [1, 3, 40, 130])
def test_nothing_that_is_masked_gets_into_a_row(gpu, rows):
    """Blocks that hold no number, behind the window, after the last token and in pages that nobody has."""
    torch, _ = gpu
    c = Cache(gpu, 2, 2, 128, torch.float16, 8, 40)
    c.append(400, [400, 330])
    q = torch.randn((2, rows, 8, 128), generator=c.gen).half().cuda()
    window = 60
    out, lse = attend(gpu, c, q, None, window)
    used = torch.zeros(c.pages, dtype=torch.bool)
    for s, n in enumerate((400, 330)):
        used[c.table_host[s, max(0, n - rows - window + 1) // 64 : (n - 1) // 64 + 1].long()] = True
    c.scales[~used.cuda()] = math.nan
    for s, n in enumerate((400, 330)):
        c.table[s, (n - 1) // 64 + 1 :] = 1 << 30
    last = int(c.table_host[0, 6])
    c.codes[last, :, 0, 16:] = 255                     # after the last token
    again, lse_again = attend(gpu, c, q, None, window)
    assert out.equal(again) and lse.equal(lse_again)


def test_a_block_without_numbers_reaches_the_rows_that_see_it(gpu):
    torch, _ = gpu
    c = Cache(gpu, 1, 2, 64, torch.bfloat16, 4, 41)
    c.append(256)
    q = torch.randn((1, 150, 4, 64), generator=c.gen).bfloat16().cuda()
    good, good_lse = attend(gpu, c, q, None)
    # rows are at 106 .. 255: block 2 (128 .. 191) is seen from row 22 on
    for which in (0, 1):
        scales = c.scales.clone()
        c.scales[int(c.table_host[0, 2]), 1, which] = math.nan
        out, lse = attend(gpu, c, q, None)
        c.scales.copy_(scales)
        hit = torch.zeros((150, 4), dtype=torch.bool, device="cuda")
        hit[22:, 2:] = True
        assert bool(out[0][hit].isnan().all())
        assert out[0][~hit].equal(good[0][~hit]) and lse[0][~hit].equal(good_lse[0][~hit])
        assert bool(lse[0][hit].isnan().all()) if which == 0 else lse.equal(good_lse)
    c.table[0, 2] = -7
    out, lse = attend(gpu, c, q, None)
    assert bool(out[0, 22:].isnan().all()) and out[0, :22].equal(good[0, :22])


@pytest.mark.parametrize("size", [1e-30, 1e-6, 3e4, 1e25])
def test_queries_of_any_size(gpu, size):
    """Large scores leave one token, small ones all; bf16 queries outside fp16's range."""
    torch, _ = gpu
    c = Cache(gpu, 1, 1, 128, torch.bfloat16, 3, 42)
    c.append(150)
    q = (torch.randn((1, 1, 4, 128), generator=c.gen) * size).bfloat16().cuda()
    scale = min(0.1, 1.0 / size)
    out, lse = attend(gpu, c, q, None, scale=scale)
    compare(gpu, c, q, None, 0, out, lse, scale=scale)
    out, lse = attend(gpu, c, q * 0, None, scale=scale)
    compare(gpu, c, q * 0, None, 0, out, lse, scale=scale)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_scales_that_are_not_positive(gpu, rows, scale):
    torch, _ = gpu
    c = Cache(gpu, 1, 2, 128, torch.float16, 3, 44)
    c.append(150)
    c.weights.zero_()
    q = torch.randn((1, rows, 4, 128), generator=c.gen).half().cuda()
    out, lse = attend(gpu, c, q, None, window=100, scale=scale, weigh=True)
    compare(gpu, c, q if scale >= 0 else -q, None, 100, out, lse, scale=abs(scale), weights=c.weights, before=torch.zeros(c.weights.shape))


# More rows than a few whatever the tables have room for; and those that are a few unless the tables have much of it.
MANY = [
    (8, 1, 128, "float16", [2100], None, 70, 0),           # tokens in parts
    (6, 1, 192, "bfloat16", [1100, 1030], [93, 60], 93, 0),
    (4, 1, 256, "float16", [1300], None, 140, 0),
    (4, 2, 64, "bfloat16", [1500, 30, 0, 800], [300, 30, 0, 1], 300, 300),
    (8, 2, 64, "float16", [40], None, 150, 0),             # rows before the first token see nothing
    (3, 3, 128, "bfloat16", [700], None, 600, 3),
    (64, 8, 128, "bfloat16", [2100, 40], [66, 1], 66, 100),
]
EITHER = [c for c in CASES if 64 < c[6] * (c[0] // c[1]) <= 512]


def widen(c):
    """Room for some 2.5 million tokens in the tables."""
    wide = c.torch.full((c.seqs, 40_000), -1, dtype=c.torch.int32, device="cuda")
    wide[:, : c.max_blocks] = c.table
    c.table = wide


@pytest.mark.parametrize("case,wide", [(c, False) for c in MANY] + [(c, True) for c in EITHER], ids=lambda c: "-".join(str(x) for x in c).replace(" ", "") if isinstance(c, tuple) else None)
def test_attention_of_many_rows(gpu, case, wide):
    heads, kv_heads, dim, dtype, lengths, counts, rows, window = case
    c, q = case_cache(gpu, case, 33)
    few = attend(gpu, c, q, counts, window)
    if wide:
        widen(c)
        compare(gpu, c, q, counts, window, *few)
    c.weights.zero_()
    before = c.weights.cpu()
    out, lse = attend(gpu, c, q, counts, window, weigh=True)
    compare(gpu, c, q, counts, window, out, lse, weights=c.weights, before=before)
    again, lse_again = attend(gpu, c, q, counts, window)
    assert out.equal(again) and lse.equal(lse_again)


@pytest.mark.parametrize("wide", [False, True])
def test_rows_beside_those_that_see_no_number(gpu, wide):
    """A block that holds none, with rows in sixteens of which some see it, and with more rows than a few."""
    torch, _ = gpu
    c = Cache(gpu, 1, 2, 64, torch.bfloat16, 4, 41)
    c.append(256)
    q = torch.randn((1, 150, 4, 64), generator=c.gen).bfloat16().cuda()
    if wide:
        widen(c)
    good, good_lse = attend(gpu, c, q, None)
    for which in (0, 1):
        scales = c.scales.clone()
        c.scales[int(c.table_host[0, 2]), 1, which] = math.nan
        out, lse = attend(gpu, c, q, None)
        c.scales.copy_(scales)
        hit = torch.zeros((150, 4), dtype=torch.bool, device="cuda")
        hit[22:, 2:] = True                            # rows are at 106 .. 255
        assert bool(out[0][hit].isnan().all())
        assert out[0][~hit].equal(good[0][~hit]) and lse[0][~hit].equal(good_lse[0][~hit])


@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_scales_that_are_not_positive_with_many_rows(gpu, scale):
    torch, _ = gpu
    c = Cache(gpu, 1, 2, 128, torch.float16, 3, 44)
    c.append(150)
    c.weights.zero_()
    widen(c)
    q = torch.randn((1, 40, 4, 128), generator=c.gen).half().cuda()
    out, lse = attend(gpu, c, q, None, window=100, scale=scale, weigh=True)
    compare(gpu, c, q if scale >= 0 else -q, None, 100, out, lse, scale=abs(scale), weights=c.weights, before=torch.zeros(c.weights.shape))


def test_rows_of_sequences_that_cannot_be_divided_evenly(gpu):
    """Three tiles of a head over blocks of very different numbers; workgroups that have parts of several units."""
    for seqs, heads, kv_heads in ((5, 6, 1), (21, 3, 1), (70, 2, 2)):
        lengths = [1 + 997 * (i * i + 3) % 1900 for i in range(seqs)]
        case = (heads, kv_heads, 64, "float16", lengths, None, 8 if heads == 6 else 1, 0)
        c, q = case_cache(gpu, case, 34)
        out, lse = attend(gpu, c, q, None)
        compare(gpu, c, q, None, 0, out, lse)


def test_attention_over_pages_beyond_four_gigabytes(gpu):
    torch, spqt = gpu
    pages = 36_000                                     # 8 heads, 128: 128 KB a page, 4.7 GB
    small = Cache(gpu, 1, 8, 128, torch.float16, 3, 43)
    small.append(150)
    q = torch.randn((1, 2, 16, 128), generator=small.gen).half().cuda()
    out, lse = attend(gpu, small, q, None)
    codes, scales, _, weights = spqt.new_kv_cache(pages, 8, 128, 1, torch.float16, True)
    far = torch.tensor([[pages - 1, 33_333, pages - 2]], dtype=torch.int32, device="cuda")
    codes[far[0].long()] = small.codes[small.table[0].long()]
    scales[far[0].long()] = small.scales[small.table[0].long()]
    small.codes, small.scales, small.weights, small.table = codes, scales, weights, far
    again, lse_again = attend(gpu, small, q, None, weigh=True)
    assert out.equal(again) and lse.equal(lse_again)
    assert float(weights[far[0].long()].sum()) == pytest.approx(2 * 16, rel=1e-5)
    # and an append there
    small.append(10)
    k, v = (torch.zeros((1, 160, 8, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    spqt.spqt_kv_read(codes, scales, far, small.lengths, k, v)
    want, scale = oracle.quantize(small.tokens[0][0][128:160, 5].double())
    assert torch.equal(k[0, 128:, 5].cpu(), oracle.rounded(want.double() * scale, torch.float16))


EVICTIONS = [
    # kv heads, dim, type, lengths, keep, recent
    (1, 64, "float16", [1], 1, 0),
    (2, 128, "float16", [200, 64, 0], 64, 10),
    (3, 128, "bfloat16", [300, 129, 65], 100, 100),
    (1, 256, "bfloat16", [500, 77], 130, 1),
    (2, 192, "float16", [190, 500], 250, 7),
    (8, 64, "float16", [3000, 2049, 1024], 1111, 64),
    (1, 128, "float16", [1025], 1024, 0),
    (1, 64, "bfloat16", [40000, 33001], 5000, 100),    # more than the selection holds in shared memory
]


@pytest.mark.parametrize("kind", ["spread", "ties", "strange"])
@pytest.mark.parametrize("case", EVICTIONS, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_eviction(gpu, case, kind):
    torch, spqt = gpu
    kv_heads, dim, dtype, lengths, keep, recent = case
    dtype = getattr(torch, dtype)
    seqs, new_blocks = len(lengths), -(-keep // 64) + 1
    blocks = max(1, -(-max(lengths) // 64))
    c = Cache(gpu, seqs, kv_heads, dim, dtype, blocks + new_blocks, 50)
    c.append(max(1, max(lengths)), lengths)
    w = torch.exp(3 * torch.randn(c.weights.shape, generator=c.gen))
    if kind == "ties":
        w = torch.floor(w).clamp(max=2)
    if kind == "strange":
        pick = torch.randint(0, 8, w.shape, generator=c.gen)
        for i, x in enumerate((math.nan, math.inf, 0.0, -0.0, -1.0, 1e-42)):
            w[pick == i] = x
    c.weights.copy_(w)
    new_table = c.table[:, blocks:].contiguous()
    old = c.table[:, :blocks].contiguous()
    new_lengths = torch.full((seqs,), 99, dtype=torch.int32, device="cuda")
    kept = torch.full((seqs, kv_heads, keep), 99, dtype=torch.int32, device="cuda")
    before = c.state()
    spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, old, c.lengths, keep, recent, new_table, new_lengths, kept)
    codes, scales, tail, weights = c.state()
    assert new_lengths.tolist() == [min(n, keep) for n in lengths]
    touched = torch.zeros(c.pages, dtype=torch.bool)
    for s, n in enumerate(lengths):
        total = min(n, keep)
        row = old[s].cpu()
        for h in range(kv_heads):
            at = before[3][row.long(), h].reshape(-1)[:n]
            want = oracle.choose(at, n, keep, recent)
            assert kept[s, h].tolist() == want + [-1] * (keep - total)
            index = torch.tensor(want, dtype=torch.long)
            for which in (0, 1):
                held = oracle.rounded(oracle.token_values(before[0], before[1], row, h, which, n)[index], dtype)
                for b in range(-(-total // 64)):
                    page, here = int(new_table[s, b]), min(64, total - 64 * b)
                    touched[page] = True
                    expected, scale = oracle.quantize(held[64 * b : 64 * b + here].double())
                    assert float(scales[page, h, which]) == scale
                    assert torch.equal(oracle.page_codes(codes[page, h], which)[:here], expected)
                    moved = torch.zeros(64)
                    moved[:here] = at[index[64 * b : 64 * b + here]]
                    assert torch.equal(weights[page, h].view(torch.int32), moved.view(torch.int32))
                if total % 64:
                    assert torch.equal(tail[s, h, which, : total % 64].view(torch.int16), held[total // 64 * 64 :].view(torch.int16))
    assert torch.equal(codes[~touched], before[0][~touched])
    for now, then in ((scales, before[1]), (weights, before[3])):
        assert torch.equal(now.view(torch.int32)[~touched], then.view(torch.int32)[~touched])


def test_evicted_sequences_go_on(gpu):
    """Append, attend, evict, append, attend: the heads then hold other tokens, at the same length."""
    torch, spqt = gpu
    c = Cache(gpu, 2, 2, 64, torch.float16, 8, 60)
    c.append(200, [200, 90])
    c.weights.zero_()
    q = torch.randn((2, 4, 4, 64), generator=c.gen).half().cuda()
    out, lse = attend(gpu, c, q, None, weigh=True)
    before = torch.zeros(c.weights.shape)
    compare(gpu, c, q, None, 0, out, lse, weights=c.weights, before=before)
    new_lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda")
    spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, c.table[:, :4].contiguous(), c.lengths, 100, 20, c.table[:, 4:].contiguous(), new_lengths, kept)
    c.table, c.table_host, c.lengths, c.length_of = c.table[:, 4:].contiguous(), c.table_host[:, 4:], new_lengths, [100, 90]
    c.max_blocks = 4
    c.append(70, [70, 3])
    assert c.lengths.tolist() == [170, 93]
    out, lse = attend(gpu, c, q, None)
    compare(gpu, c, q, None, 0, out, lse)


def test_a_decode_step_in_a_graph(gpu):
    """lengths += 1, append, attention with weights, captured once and replayed with eager work in between, against eager calls."""
    torch, spqt = gpu
    results = []
    for graphed in (False, True):
        c = Cache(gpu, 3, 2, 128, torch.float16, 5, 70)
        c.append(130, [130, 61, 1])
        ws = spqt.new_kv_workspace(3, 1, 8, 2, 128, 5)
        x = torch.zeros((3, 1, 12, 128), dtype=torch.float16, device="cuda")
        out, lse = torch.zeros((3, 1, 8, 128), dtype=torch.float16, device="cuda"), torch.zeros((3, 1, 8), device="cuda")

        def step():
            c.lengths.add_(1)
            spqt.spqt_kv_append(c.codes, c.scales, c.tail, c.table, c.lengths, x[:, :, 8:10], x[:, :, 10:], weights=c.weights)
            spqt.spqt_kv_attention(c.codes, c.scales, c.table, c.lengths, x[:, :, :8], out, ws, lse=lse, weights=c.weights, decay=0.9)

        graph = None
        if graphed:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        seen = []
        for i in range(6):
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(100 + i)).half())
            step() if graph is None else graph.replay()
            torch.cuda.synchronize()
            seen.append((out.clone(), lse.clone(), c.weights.clone()))
            out.fill_(5.0)
        results.append(seen)
    for eager, replayed in zip(*results):
        for a, b in zip(eager, replayed):
            assert a.equal(b)


def test_another_stream_and_a_shared_workspace(gpu):
    torch, spqt = gpu
    c, q = case_cache(gpu, CASES[7], 80)
    d, p = case_cache(gpu, CASES[9], 81)
    ws = spqt.new_kv_workspace(3, 64, 64, 8, 128, 64)
    want = [attend(gpu, *a) for a in ((c, q, None), (d, p, [5, 1, 3]))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        for handle in (side, side.cuda_stream):
            got = []
            side.wait_stream(torch.cuda.current_stream())
            for a in ((c, q, None), (d, p, [5, 1, 3])):
                with torch.cuda.stream(side):
                    got.append(attend(gpu, *a, stream=handle, workspace=ws))
            side.synchronize()
            for x, y in zip(want, got):
                assert x[0].equal(y[0]) and x[1].equal(y[1])


def test_one_workspace_for_calls_of_all_shapes(gpu):
    """Counters lie where every shape looks for them, and partial sums of one call are not in the way of the next."""
    torch, spqt = gpu
    cases = [CASES[i] for i in (7, 18, 3, 19, 8, 21, 9, 11)]
    made = [case_cache(gpu, case, 82) for case in cases]
    ws = max((spqt.new_kv_workspace(4, 4096, 64, 1, dim, 64) for dim in (64, 128, 192, 256)), key=lambda w: w.numel())
    for _ in range(2):
        for case, (c, q) in zip(cases, made):
            want = attend(gpu, c, q, case[5], case[7])
            got = attend(gpu, c, q, case[5], case[7], workspace=ws)
            assert want[0].equal(got[0]) and want[1].equal(got[1])


def test_through_the_extension_module_and_without_it(gpu, monkeypatch):
    """The same results bit for bit, also on a stream that torch has made current."""
    torch, spqt = gpu
    from paper_2511_04477_amd import binding
    assert binding._fast is not None
    side = torch.cuda.Stream()
    results = []
    for fast, stream in ((True, torch.cuda.current_stream()), (False, torch.cuda.current_stream()), (True, side), (False, side)):
        with monkeypatch.context() as m:
            if not fast:
                m.setattr(binding, "_fast", None)
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                c = Cache(gpu, 2, 2, 64, torch.bfloat16, 8, 90)
                c.codes.fill_(128)                     # the pool's bytes that no token writes
                c.append(200, [200, 90])
                q = torch.randn((2, 3, 4, 64), generator=c.gen).bfloat16().cuda()
                out, lse = attend(gpu, c, q, None, window=150, weigh=True, decay=0.5)
                new_lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
                kept = torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda")
                spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, c.table[:, :4].contiguous(), c.lengths, 100, 20, c.table[:, 4:].contiguous(), new_lengths, kept)
                k, v = (torch.zeros((2, 100, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
                spqt.spqt_kv_read(c.codes, c.scales, c.table[:, 4:].contiguous(), new_lengths, k, v, counts=new_lengths)
                results.append((out, lse, kept, k, v, c.weights))
            stream.synchronize()
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert a.equal(b)


@pytest.mark.parametrize("fast", [True, False])
def test_refusals(gpu, fast, monkeypatch):
    torch, spqt = gpu
    if not fast:
        from paper_2511_04477_amd import binding
        monkeypatch.setattr(binding, "_fast", None)
    c, q = case_cache(gpu, CASES[2], 90)
    ws = spqt.new_kv_workspace(3, 1, 8, 2, 128, 4)
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    good = dict(codes=c.codes, scales=c.scales, table=c.table, lengths=c.lengths, q=q, out=out, workspace=ws)
    spqt.spqt_kv_attention(**good)
    wide = torch.zeros((3, 1, 8, 256), dtype=q.dtype, device="cuda")
    for bad in (dict(codes=c.codes.cpu()), dict(codes=c.codes.view(torch.int8)), dict(scales=c.scales.double()), dict(scales=c.scales[1:]), dict(table=c.table.long()),
                dict(table=c.table[0]), dict(lengths=c.lengths[:2]), dict(lengths=c.lengths.float()), dict(q=q.float()), dict(q=q[0]), dict(q=q[:2]), dict(q=q[:, :, :7]),
                dict(q=q[..., :64]), dict(out=out[..., ::2]), dict(out=out.half()), dict(out=out[:, :, 1:]), dict(out=wide[..., ::2]), dict(out=wide[..., 1:129]),
                dict(workspace=ws[:100]), dict(workspace=None), dict(counts=c.lengths[:1]), dict(counts=c.lengths.long()), dict(window=-1), dict(weights=c.weights),
                dict(lse=torch.zeros((3, 1, 7), device="cuda")), dict(weights=c.weights[1:], lse=torch.zeros((3, 1, 8), device="cuda")), dict(scale=float("nan"))):
        with pytest.raises(spqt.SpqtError):
            spqt.spqt_kv_attention(**dict(good, **bad))
    x = torch.zeros((3, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    good = dict(codes=c.codes, scales=c.scales, tail=c.tail, table=c.table, lengths=c.lengths, k=x, v=x)
    for bad in (dict(tail=c.tail.half()), dict(tail=c.tail[:1]), dict(tail=None), dict(k=x.float()), dict(k=x[:, :, :1]), dict(v=x.half()), dict(v=x[:, :0]), dict(k=x[:, :0], v=x[:, :0]),
                dict(weights=c.weights[1:])):
        with pytest.raises(spqt.SpqtError):
            spqt.spqt_kv_append(**dict(good, **bad))
    kept, new_lengths = torch.zeros((3, 2, 64), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    good = dict(codes=c.codes, scales=c.scales, tail=c.tail, weights=c.weights, table=c.table[:, :2].contiguous(), lengths=c.lengths, keep=64, recent=3,
                new_table=c.table[:, 2:].contiguous(), new_lengths=new_lengths, kept=kept)
    for bad in (dict(weights=None), dict(keep=63), dict(recent=65), dict(recent=-1), dict(new_lengths=c.lengths), dict(kept=kept.float()), dict(new_table=c.table[0]),
                dict(new_table=c.table[:, :0].contiguous())):
        with pytest.raises(spqt.SpqtError):
            spqt.spqt_kv_evict(**dict(good, **bad))
