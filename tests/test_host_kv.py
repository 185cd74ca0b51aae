"""The key/value cache's entry points on the host: what the header declares is exported, and what is refused is refused before
anything is launched."""
import ctypes

import pytest

import paper_2511_04477_amd as spqt
from paper_2511_04477_amd.kv import KvCacheView, KvRowsView
from test_host import declared_functions

EINVAL, ESHAPE, EALIGN, ESIZE = -1, -2, -3, -4


def test_header_symbols_are_exported():
    names = [n for n in declared_functions("spqt_kv.h") if n.startswith("spqt_kv")]
    assert set(names) == set(spqt.KV_EXPORTS)
    for n in names:
        assert getattr(spqt.lib(), n) is not None


def cache(**more):
    given = dict(codes=1 << 20, scales=1 << 20, tail=1 << 20, weights=None, table=1 << 20, lengths=1 << 20, pages=4, sequences=2, max_blocks=2, kv_heads=2,
                 head_dim=128, type=0)
    given.update(more)
    return KvCacheView(*(given[f] for f, _ in KvCacheView._fields_))


def rows(data=1 << 20, sequence=256, row=256, head=128):
    return KvRowsView(data, sequence, row, head)


BAD_CACHES = [(dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(table=None), EINVAL), (dict(lengths=None), EINVAL), (dict(type=2), EINVAL),
              (dict(pages=0), ESHAPE), (dict(pages=1 << 31), ESHAPE), (dict(sequences=0), ESHAPE), (dict(sequences=65536), ESHAPE), (dict(max_blocks=0), ESHAPE),
              (dict(kv_heads=0), ESHAPE), (dict(kv_heads=16385), ESHAPE), (dict(head_dim=96), ESHAPE), (dict(head_dim=0), ESHAPE), (dict(head_dim=320), ESHAPE),
              (dict(codes=(1 << 20) + 8), EALIGN), (dict(scales=(1 << 20) + 4), EALIGN), (dict(table=(1 << 20) + 2), EALIGN), (dict(weights=(1 << 20) + 4), EALIGN)]
BAD_ROWS = [(dict(data=None), EINVAL), (dict(head=-8), EINVAL), (dict(data=(1 << 20) + 2), EALIGN), (dict(row=132), EALIGN)]


def append(c, k, v, n=1):
    return spqt.lib().spqt_kv_append(ctypes.byref(c), ctypes.byref(k), ctypes.byref(v), n, None, None)


def read(c, k, v, n=1):
    return spqt.lib().spqt_kv_read(ctypes.byref(c), ctypes.byref(k), ctypes.byref(v), n, None, None)


def attention(c, q, out, n=1, lse=None, heads=4, scale=0.1, window=0, decay=1.0, ws=1 << 20, size=1 << 40):
    return spqt.lib().spqt_kv_attention(ctypes.byref(c), ctypes.byref(q), ctypes.byref(out), lse, n, None, heads, scale, window, decay, ws, size, None)


def evict(c, keep=64, recent=1, table=1 << 21, blocks=2, lengths=1 << 21, kept=1 << 20):
    return spqt.lib().spqt_kv_evict(ctypes.byref(c), keep, recent, table, blocks, lengths, kept, None)


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches_that_are_refused(bad, status):
    assert append(cache(**bad), rows(), rows()) == status
    assert read(cache(**bad), rows(), rows()) == status
    assert attention(cache(**bad), rows(), rows()) == status
    assert evict(cache(**dict(dict(weights=1 << 20), **bad))) == status


@pytest.mark.parametrize("bad,status", BAD_ROWS)
def test_rows_that_are_refused(bad, status):
    for call in (append, read, attention):
        assert call(cache(), rows(**bad), rows()) == status
        assert call(cache(), rows(), rows(**bad)) == status
        assert call(cache(), rows(), rows(), 0) == ESHAPE
        assert call(cache(), rows(), rows(), (1 << 24) + 1) == ESHAPE


def test_append_needs_a_tail():
    assert append(cache(tail=None), rows(), rows()) == EINVAL
    assert append(cache(tail=(1 << 20) + 4), rows(), rows()) == EALIGN


@pytest.mark.parametrize("bad,status", [(dict(heads=3), ESHAPE), (dict(heads=1), ESHAPE), (dict(heads=0), ESHAPE), (dict(window=-1), EINVAL),
                                        (dict(scale=float("nan")), EINVAL), (dict(decay=float("nan")), EINVAL), (dict(ws=None), EINVAL),
                                        (dict(ws=(1 << 20) + 16), EALIGN), (dict(lse=(1 << 20) + 2), EALIGN), (dict(size=16), ESIZE)])
def test_attention_that_is_refused(bad, status):
    assert attention(cache(), rows(), rows(), **bad) == status


def test_weights_need_lse():
    assert attention(cache(weights=1 << 20), rows(), rows()) == EINVAL


@pytest.mark.parametrize("bad,status", [(dict(keep=0), EINVAL), (dict(recent=-1), EINVAL), (dict(recent=65), EINVAL), (dict(keep=129), ESHAPE),
                                        (dict(blocks=0), ESHAPE), (dict(table=None), EINVAL), (dict(lengths=None), EINVAL), (dict(kept=None), EINVAL),
                                        (dict(lengths=1 << 20), EINVAL), (dict(table=1 << 20), EINVAL), (dict(kept=(1 << 20) + 2), EALIGN)])
def test_eviction_that_is_refused(bad, status):
    assert evict(cache(weights=1 << 20), **bad) == status


def test_eviction_needs_weights_and_a_tail():
    assert evict(cache()) == EINVAL
    assert evict(cache(weights=1 << 20, tail=None)) == EINVAL


def test_workspace_sizes():
    out = ctypes.c_size_t()
    size = spqt.spqt_kv_workspace_bytes
    assert size(1, 1, 8, 8, 128, 1) >= 256 and size(3, 5, 40, 8, 256, 4096) >= size(1, 1, 8, 8, 64, 1)
    L = spqt.lib()
    assert L.spqt_kv_workspace_bytes(1, 1, 8, 8, 128, 1, None) == EINVAL
    for bad in [(0, 1, 8, 8, 128, 1), (1, 0, 8, 8, 128, 1), (1, 1, 9, 8, 128, 1), (1, 1, 8, 8, 100, 1), (1, 1, 8, 8, 128, 0)]:
        assert L.spqt_kv_workspace_bytes(*bad, ctypes.byref(out)) == ESHAPE
        with pytest.raises(spqt.SpqtError):
            size(*bad)


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
def test_a_workspace_for_more_serves_less(dim):
    size = spqt.spqt_kv_workspace_bytes
    steps = [1, 3, 16, 64, 65, 200, 512, 513, 4000]
    for sequences in (1, 5, 300):
        for blocks in (1, 7, 8, 400, 100_000):
            sizes = [size(sequences, rows, 8, 8, dim, blocks) for rows in steps]
            assert sizes == sorted(sizes)
            assert sizes == [size(1, rows, 8, 8, dim, 1) for rows in steps]


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    codes, scales = torch.zeros((2, 1, 2, 64, 64), dtype=torch.uint8), torch.zeros((2, 1, 2))
    table, lengths = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros((1, 1, 1, 64), dtype=torch.float16)
    for call in (lambda: spqt.spqt_kv_append(codes, scales, x, table, lengths, x, x), lambda: spqt.spqt_kv_read(codes, scales, table, lengths, x, x),
                 lambda: spqt.spqt_kv_attention(codes, scales, table, lengths, x, x, codes), lambda: spqt.spqt_kv_attention(codes, scales, table, lengths, None, x, codes),
                 lambda: spqt.spqt_kv_evict(codes, scales, x, scales, table, lengths, 4, 1, table, lengths, table)):
        with pytest.raises(spqt.SpqtError):
            call()
    with pytest.raises(spqt.SpqtError):
        spqt.new_kv_cache(4, 2, 96, 1)
