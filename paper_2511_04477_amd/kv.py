"""The key/value cache in 8 bits: binding of include/spqt_kv.h, in the manner of binding.py.

A cache is a handful of tensors that the caller owns (`new_kv_cache` makes them):

    codes   uint8 [pages, kv_heads, 2, 64, head_dim]     scales  float32 [pages, kv_heads, 2]
    table   int32 [sequences, max_blocks]                lengths int32 [sequences]
    tail    float16 or bfloat16 [sequences, kv_heads, 2, 64, head_dim]
    weights float32 [pages, kv_heads, 64], where attention is to count what tokens weigh

`lengths` count the tokens of the call: a decode step adds them first (`lengths += 1`), once for all layers.  16-bit
tensors [sequences, rows, heads, head_dim] may be slices of a larger one as long as the last dimension is dense and the
strides are multiples of 8.  `counts`, int32 [sequences], says how many of a call's rows a sequence has (None: all).

Lengths are never merely set back: to take tokens back (drafts that were rejected), put back the codes and scales of the page
that was open before their append, and the sequence's tail, from copies made then, and the lengths after that.
"""
from __future__ import annotations

import ctypes

from . import binding as _b
from .binding import KV_EXPORTS, SpqtError, _check, lib  # noqa: F401

KV_BLOCK = 64


class KvCacheView(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("tail", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("pages", ctypes.c_int64), ("sequences", ctypes.c_int), ("max_blocks", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("type", ctypes.c_int)]


class KvRowsView(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("sequence", ctypes.c_int64), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


def _int32(v, what):
    """v as an int that a C int holds; ctypes would keep the lowest 32 bits of any other."""
    try:
        n = int(v)
    except (TypeError, ValueError, OverflowError):
        raise SpqtError(f"{what}: need an integer") from None
    if not -(1 << 31) <= n < 1 << 31:
        raise SpqtError(f"{what}: {n} is beyond 32 bits")
    return n


def _tensor(t, dtype, shape, what, device=None):
    """Device pointer of a contiguous tensor; None in the shape stands for any extent."""
    if not (isinstance(t, _b._torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise SpqtError(f"{what}: need a contiguous CUDA tensor of dtype {dtype}")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise SpqtError(f"{what}: shape {tuple(t.shape)} does not match {shape}")
    if device is not None and t.device != device:
        raise SpqtError(f"{what}: on {t.device}, the cache is on {device}")
    return t.data_ptr()


def _rows(t, dtype, shape, what, device):
    if not (isinstance(t, _b._torch.Tensor) and t.is_cuda and t.dtype == dtype and t.dim() == 4):
        raise SpqtError(f"{what}: need a CUDA tensor [sequences, rows, heads, head_dim] of dtype {dtype}")
    if any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise SpqtError(f"{what}: shape {tuple(t.shape)} does not match {shape}")
    if t.device != device:
        raise SpqtError(f"{what}: on {t.device}, the cache is on {device}")
    if t.stride(3) != 1:
        raise SpqtError(f"{what}: the last dimension has to be dense")
    return KvRowsView(t.data_ptr(), *(t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)))


def _cache(codes, scales, table, lengths, dtype, tail=None, weights=None):
    torch = _b._torch or _b._load_torch()
    if dtype not in (torch.float16, torch.bfloat16):
        raise SpqtError("the 16-bit tensors have to be float16 or bfloat16")
    cp = _tensor(codes, torch.uint8, (None, None, 2, KV_BLOCK, None), "codes")
    pages, heads, _, _, dim = codes.shape
    tp = _tensor(table, torch.int32, (None, None), "table", codes.device)
    sequences, blocks = table.shape
    return KvCacheView(cp, _tensor(scales, torch.float32, (pages, heads, 2), "scales", codes.device),
                       None if tail is None else _tensor(tail, dtype, (sequences, heads, 2, KV_BLOCK, dim), "tail", codes.device),
                       None if weights is None else _tensor(weights, torch.float32, (pages, heads, KV_BLOCK), "weights", codes.device),
                       tp, _tensor(lengths, torch.int32, (sequences,), "lengths", codes.device), pages, _int32(sequences, "sequences"), _int32(blocks, "blocks of the table"),
                       _int32(heads, "kv heads"), _int32(dim, "head_dim"),
                       1 if dtype == torch.bfloat16 else 0)


def _counts(counts, cache, device):
    return None if counts is None else _tensor(counts, _b._torch.int32, (cache.sequences,), "counts", device)


def _dtype_of(t, what):
    torch = _b._torch or _b._load_torch()
    if not isinstance(t, torch.Tensor):
        raise SpqtError(f"{what}: need a CUDA tensor")
    return t.dtype


def new_kv_cache(pages: int, kv_heads: int, head_dim: int, sequences: int, dtype=None, weights: bool = False, device="cuda"):
    """(codes, scales, tail, weights or None) of an empty cache of one layer; table and lengths are the caller's, shared by all layers."""
    torch = _b._torch or _b._load_torch()
    dtype = torch.float16 if dtype is None else dtype
    if head_dim not in (64, 128, 192, 256) or min(pages, kv_heads, sequences) < 1 or dtype not in (torch.float16, torch.bfloat16):
        raise SpqtError("new_kv_cache: head_dim is 64, 128, 192 or 256, dtype float16 or bfloat16, and the extents are at least 1")
    return (torch.empty((pages, kv_heads, 2, KV_BLOCK, head_dim), dtype=torch.uint8, device=device),
            torch.empty((pages, kv_heads, 2), dtype=torch.float32, device=device),
            torch.empty((sequences, kv_heads, 2, KV_BLOCK, head_dim), dtype=dtype, device=device),
            torch.zeros((pages, kv_heads, KV_BLOCK), dtype=torch.float32, device=device) if weights else None)


def spqt_kv_append(codes, scales, tail, table, lengths, k, v, counts=None, weights=None, stream=None) -> None:
    """Quantizes k and v [sequences, rows, kv_heads, head_dim] into the cache as the last counts[s] of lengths[s] tokens, which follow those of earlier calls."""
    if _b._fast is not None:
        rc = _b._fast.kv_append((_b._lib or lib()).at["spqt_kv_append"], codes, scales, tail, table, lengths, k, v, counts, weights, stream)
        if rc is not None:
            return _check(rc)
    dtype = _dtype_of(k, "k")
    cache = _cache(codes, scales, table, lengths, dtype, tail, weights)
    shape = (cache.sequences, None, cache.kv_heads, cache.head_dim)
    keys, values = _rows(k, dtype, shape, "k", codes.device), _rows(v, dtype, (cache.sequences, k.shape[1]) + shape[2:], "v", codes.device)
    _check(lib().spqt_kv_append(ctypes.byref(cache), ctypes.byref(keys), ctypes.byref(values), _int32(k.shape[1], "rows"), _counts(counts, cache, codes.device),
                                _b._stream_ptr(stream)))


def spqt_kv_read(codes, scales, table, lengths, k_out, v_out, counts=None, stream=None) -> None:
    """The last counts[s] tokens of every sequence as 16-bit values, into k_out and v_out [sequences, rows, kv_heads, head_dim]; other rows are set to 0."""
    if _b._fast is not None:
        rc = _b._fast.kv_read((_b._lib or lib()).at["spqt_kv_read"], codes, scales, table, lengths, k_out, v_out, counts, stream)
        if rc is not None:
            return _check(rc)
    dtype = _dtype_of(k_out, "k_out")
    cache = _cache(codes, scales, table, lengths, dtype)
    shape = (cache.sequences, None, cache.kv_heads, cache.head_dim)
    keys, values = _rows(k_out, dtype, shape, "k_out", codes.device), _rows(v_out, dtype, (cache.sequences, k_out.shape[1]) + shape[2:], "v_out", codes.device)
    _check(lib().spqt_kv_read(ctypes.byref(cache), ctypes.byref(keys), ctypes.byref(values), _int32(k_out.shape[1], "rows"), _counts(counts, cache, codes.device),
                              _b._stream_ptr(stream)))


def spqt_kv_workspace_bytes(sequences: int, rows: int, q_heads: int, kv_heads: int, head_dim: int, max_blocks: int) -> int:
    out = ctypes.c_size_t()
    sizes = [_int32(n, "spqt_kv_workspace_bytes") for n in (sequences, rows, q_heads, kv_heads, head_dim, max_blocks)]
    _check(lib().spqt_kv_workspace_bytes(*sizes, ctypes.byref(out)))
    return out.value


def new_kv_workspace(sequences: int, rows: int, q_heads: int, kv_heads: int, head_dim: int, max_blocks: int, device="cuda"):
    """Allocate and prepare a workspace tensor for spqt_kv_attention with up to this many rows; attention calls of one stream may share it, GEMVs may not."""
    torch = _b._torch or _b._load_torch()
    ws = torch.empty(spqt_kv_workspace_bytes(sequences, rows, q_heads, kv_heads, head_dim, max_blocks), dtype=torch.uint8, device=device)
    _b.spqt_workspace_init(ws)
    return ws


def spqt_kv_attention(codes, scales, table, lengths, q, out, workspace, scale=None, counts=None, window: int = 0, lse=None, weights=None, decay: float = 1.0,
                      stream=None) -> None:
    """Attention of q [sequences, rows, q_heads, head_dim] over the cache into out (same shape and type): row i is the token at position
    lengths[s] - counts[s] + i and sees those up to itself, the last `window` of them if window > 0.  scale None: 1 / sqrt(head_dim).
    lse: float32 [sequences, rows, q_heads] or None.  weights (with lse): weights = decay * weights + the probabilities that every
    cached token got in this call.  out may be q itself in calls without weights."""
    if _b._fast is not None:
        rc = _b._fast.kv_attention((_b._lib or lib()).at["spqt_kv_attention"], codes, scales, table, lengths, q, out, workspace, scale, counts, window, lse, weights, decay, stream)
        if rc is not None:
            return _check(rc)
    dtype = _dtype_of(q, "q")
    cache = _cache(codes, scales, table, lengths, dtype, None, weights)
    device = codes.device
    qv = _rows(q, dtype, (cache.sequences, None, None, cache.head_dim), "q", device)
    ov = _rows(out, dtype, tuple(q.shape), "out", device)
    lp = None if lse is None else _tensor(lse, _b._torch.float32, tuple(q.shape[:3]), "lse", device)
    wp = _tensor(workspace, _b._torch.uint8, (None,), "workspace", device)
    if scale is None:
        scale = cache.head_dim ** -0.5
    _check(lib().spqt_kv_attention(ctypes.byref(cache), ctypes.byref(qv), ctypes.byref(ov), lp, _int32(q.shape[1], "rows"), _counts(counts, cache, device),
                                   _int32(q.shape[2], "q heads"), float(scale), _int32(window, "window"), float(decay), wp, workspace.numel(), _b._stream_ptr(stream)))


def spqt_kv_evict(codes, scales, tail, weights, table, lengths, keep: int, recent: int, new_table, new_lengths, kept, stream=None, exact: bool = False) -> None:
    """Cuts every sequence down to `keep` tokens per kv head, the last `recent` ones and the heaviest others, and moves them to the pages
    of new_table int32 [sequences, new_blocks].  new_lengths int32 [sequences] and kept int32 [sequences, kv_heads, keep] are written.
    exact: tokens move without a rounding to 16 bits in between (spqt_kv_evict_exact), as caches that are cut down again and again need it."""
    name = "spqt_kv_evict_exact" if exact else "spqt_kv_evict"
    if _b._fast is not None:
        rc = _b._fast.kv_evict((_b._lib or lib()).at[name], codes, scales, tail, weights, table, lengths, keep, recent, new_table, new_lengths, kept, stream)
        if rc is not None:
            return _check(rc)
    torch = _b._torch or _b._load_torch()
    cache = _cache(codes, scales, table, lengths, _dtype_of(tail, "tail"), tail, weights)
    device = codes.device
    np_ = _tensor(new_table, torch.int32, (cache.sequences, None), "new_table", device)
    lp = _tensor(new_lengths, torch.int32, (cache.sequences,), "new_lengths", device)
    keep, recent = _int32(keep, "keep"), _int32(recent, "recent")
    kp = _tensor(kept, torch.int32, (cache.sequences, cache.kv_heads, keep), "kept", device)
    _check(getattr(lib(), name)(ctypes.byref(cache), keep, recent, np_, _int32(new_table.shape[1], "blocks of new_table"), lp, kp, _b._stream_ptr(stream)))
