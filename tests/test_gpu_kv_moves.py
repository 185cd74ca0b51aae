"""The exact eviction on the GPU against the 64-bit oracle, bit for bit, once and again and again."""
import math

import pytest
import torch

from oracle import kv as oracle
from test_gpu_kv import Cache, EVICTIONS, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["spread", "ties"])
@pytest.mark.parametrize("case", EVICTIONS, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_exact_eviction(gpu, case, kind):  # noqa: F811
    _, spqt = gpu
    kv_heads, dim, dtype, lengths, keep, recent = case
    dtype = getattr(torch, dtype)
    seqs, new_blocks = len(lengths), -(-keep // 64) + 1
    blocks = max(1, -(-max(lengths) // 64))
    c = Cache(gpu, seqs, kv_heads, dim, dtype, blocks + new_blocks, 51)
    c.append(max(1, max(lengths)), lengths, x=c.values(max(1, max(lengths)), 2.0))
    w = torch.exp(3 * torch.randn(c.weights.shape, generator=c.gen))
    c.weights.copy_(torch.floor(w).clamp(max=2) if kind == "ties" else w)
    new_table, old = c.table[:, blocks:].contiguous(), c.table[:, :blocks].contiguous()
    new_lengths = torch.full((seqs,), 99, dtype=torch.int32, device="cuda")
    kept = torch.full((seqs, kv_heads, keep), 99, dtype=torch.int32, device="cuda")
    before = c.state()
    spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, old, c.lengths, keep, recent, new_table, new_lengths, kept, exact=True)
    codes, scales, tail, weights = c.state()
    assert new_lengths.tolist() == [min(n, keep) for n in lengths]
    touched = torch.zeros(c.pages, dtype=torch.bool)
    for s, n in enumerate(lengths):
        total, row = min(n, keep), old[s].cpu()
        for h in range(kv_heads):
            at = before[3][row.long(), h].reshape(-1)[:n]
            want = oracle.choose(at, n, keep, recent)
            assert kept[s, h].tolist() == want + [-1] * (keep - total)
            for b in range(-(-total // 64)):
                page, here = int(new_table[s, b]), want[64 * b : min(total, 64 * b + 64)]
                touched[page] = True
                for which in (0, 1):
                    parts = []
                    for block in sorted({t // 64 for t in here}):
                        rows = [t % 64 for t in here if t // 64 == block]
                        parts.append((oracle.page_codes(before[0][row[block], h], which)[rows], float(before[1][row[block], h, which])))
                    expected, scale = oracle.requantize(parts)
                    assert float(scales[page, h, which]) == scale
                    assert torch.equal(oracle.page_codes(codes[page, h], which)[: len(here)], expected)
                    if len(here) < 64:
                        held = oracle.rounded(expected.double() * scale, dtype)
                        assert torch.equal(tail[s, h, which, : len(here)].view(torch.int16), held.view(torch.int16))
                moved = torch.zeros(64)
                moved[: len(here)] = at[torch.tensor(here, dtype=torch.long)]
                assert torch.equal(weights[page, h], moved)
    assert torch.equal(codes[~touched], before[0][~touched])
    for now, then in ((scales, before[1]), (weights, before[3])):
        assert torch.equal(now.view(torch.int32)[~touched], then.view(torch.int32)[~touched])


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
def test_what_always_stays_never_changes(gpu, dtype, dim):  # noqa: F811
    """Forty evictions, each with fresh tokens appended and dropped again: the blocks in front are as they were, and an open block that only moves, too."""
    _, spqt = gpu
    heads, stay = 2, 300                                     # tokens that weigh most: four blocks and a part of one
    c = Cache(gpu, 1, heads, dim, getattr(torch, dtype), 14, 52)
    tables = [c.table[:, :7].contiguous(), c.table[:, 7:].contiguous()]
    hosts = [c.table_host[:, :7], c.table_host[:, 7:]]
    c.table, c.table_host = tables[0], hosts[0]
    c.append(stay)
    c.weights.fill_(5.0)

    def held(host):
        codes, scales, tail, _ = c.state()
        pages = [int(p) for p in host[0, :5]]
        found = [[[oracle.page_codes(codes[p, h], which)[: min(64, stay - 64 * b)] for b, p in enumerate(pages)] for which in (0, 1)] for h in range(heads)]
        return found, scales[pages], tail[:, :, :, : stay % 64]

    first = held(hosts[0])
    new_lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = torch.zeros((1, heads, stay), dtype=torch.int32, device="cuda")
    for i in range(40):
        c.table, c.table_host = tables[i % 2], hosts[i % 2]
        if i > 1:
            # 50 more: the open block may take on their scale while they are there, the whole ones do not
            c.lengths.fill_(stay + 50)
            x = torch.randn((1, 50, 2 * heads, dim), generator=c.gen).to(c.dtype).cuda()
            spqt.spqt_kv_append(c.codes, c.scales, c.tail, c.table, c.lengths, x[:, :, :heads], x[:, :, heads:], weights=c.weights)
        spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, c.table, c.lengths, stay, 0, tables[1 - i % 2], new_lengths, kept, exact=True)
        assert torch.equal(kept[0].cpu(), torch.arange(stay, dtype=torch.int32).expand(heads, -1))
        c.lengths.copy_(new_lengths)
        found, scales, tail = held(hosts[1 - i % 2])
        assert torch.equal(scales[:4], first[1][:4])
        for h in range(heads):
            for which in (0, 1):
                for b in range(4):
                    assert torch.equal(found[h][which][b], first[0][h][which][b])
        if i <= 1:
            assert torch.equal(scales, first[1]) and all(torch.equal(found[h][w][4], first[0][h][w][4]) for h in range(heads) for w in (0, 1))


def test_blocks_of_zeros_and_of_no_numbers_move(gpu):  # noqa: F811
    _, spqt = gpu
    c = Cache(gpu, 1, 1, 64, torch.float16, 8, 53)
    x = c.values(192)
    x[:, :64] = 0.0
    c.append(192, x=x)
    c.scales[int(c.table_host[0, 2]), 0, 1] = math.nan
    old, new = c.table[:, :4].contiguous(), c.table[:, 4:].contiguous()
    new_lengths, kept = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, 1, 192), dtype=torch.int32, device="cuda")
    before = c.state()
    spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, old, c.lengths, 192, 0, new, new_lengths, kept, exact=True)
    codes, scales, _, _ = c.state()
    for b in range(3):
        was, now = int(old[0, b]), int(new[0, b])
        assert torch.equal(scales[now, 0, 0], before[1][was, 0, 0]) and torch.equal(codes[now, 0, 0], before[0][was, 0, 0])
        if b < 2:
            assert torch.equal(scales[now, 0, 1], before[1][was, 0, 1]) and torch.equal(codes[now, 0, 1], before[0][was, 0, 1])
    assert bool(scales[int(new[0, 2]), 0, 1].isnan())
    # kept tokens of a block of zeros beside others
    c.lengths.fill_(100)
    c.weights[int(old[0, 0])] = 1.0
    c.weights[int(old[0, 1])] = 2.0
    kept = torch.zeros((1, 1, 50), dtype=torch.int32, device="cuda")
    spqt.spqt_kv_evict(c.codes, c.scales, c.tail, c.weights, old, c.lengths, 50, 0, new, new_lengths, kept, exact=True)
    assert kept[0, 0].tolist() == list(range(14)) + list(range(64, 100))
    codes, scales, _, _ = c.state()
    page = int(new[0, 0])
    for which in (0, 1):
        parts = [(oracle.page_codes(before[0][int(old[0, b]), 0], which)[rows], float(before[1][int(old[0, b]), 0, which])) for b, rows in ((0, slice(0, 14)), (1, slice(0, 36)))]
        expected, scale = oracle.requantize(parts)
        assert float(scales[page, 0, which]) == scale and torch.equal(oracle.page_codes(codes[page, 0], which)[:50], expected)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("before,drafts", [(70, 5), (70, 90), (64, 3), (127, 1), (60, 200)])
def test_drafts_that_are_taken_back(gpu, dtype, before, drafts):  # noqa: F811
    """With the open page and the tail put back, the cache goes on as if they had never come, also with drafts that are larger and that fill the block."""
    _, spqt = gpu
    c, d = (Cache(gpu, 2, 2, 128, getattr(torch, dtype), 6, 54) for _ in range(2))
    x = c.values(before)
    for one in (c, d):
        one.append(before, [before, 1], x=x)
    pages = [int(c.table_host[0, before // 64]), int(c.table_host[1, 0])]
    saved = [t.clone() for t in (c.codes[pages], c.scales[pages], c.tail)]
    y = 20.0 * torch.randn((2, drafts, 4, 128), generator=c.gen)
    c.append(drafts, x=y.to(c.dtype))
    c.codes[pages], c.scales[pages] = saved[0], saved[1]
    c.tail.copy_(saved[2])
    c.length_of = [before, 1]
    c.tokens = [[t[s][:n] for s, n in enumerate(c.length_of)] for t in c.tokens]
    z = c.values(40, 1.0)
    for one in (c, d):
        one.append(40, x=z)
    for s, n in enumerate(c.length_of):
        for b in range(-(-n // 64)):
            page, here = int(c.table_host[s, b]), min(64, n - 64 * b)
            assert torch.equal(c.scales[page], d.scales[page])
            for h in range(2):
                for which in (0, 1):
                    assert torch.equal(oracle.page_codes(c.codes[page, h].cpu(), which)[:here], oracle.page_codes(d.codes[page, h].cpu(), which)[:here])
        assert torch.equal(c.tail[s, :, :, : n % 64].view(torch.int16), d.tail[s, :, :, : n % 64].view(torch.int16))
