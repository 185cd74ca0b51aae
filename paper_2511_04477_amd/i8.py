"""The prompt side of a decoder in 8-bit integers: binding of include/spqt_i8.h, in the manner of binding.py.

Rows of float16 or bfloat16 values [rows, K] are held as int8 codes [rows, K] and float32 scales [rows]: tokens as rows of activations,
output channels as rows of weights.  16-bit tensors may be slices of larger ones as long as the last dimension is dense; codes begin at a multiple
of 16 bytes and have rows that are a multiple of 16 bytes apart (`new_i8_codes` makes such a tensor of any width).  All tensors of
a call are on torch's current device.
"""
from __future__ import annotations

import ctypes

from . import binding as _b
from .binding import I8_EXPORTS, SpqtError, _check, lib  # noqa: F401


class I8NormCall(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("h", "block", "block_gain", "gate", "gain", "h_out", "out", "codes", "scales")]
                + [(n, ctypes.c_int64) for n in ("h_row", "block_row", "gate_row", "h_out_row", "out_row", "codes_row", "rows", "K")]
                + [(n, ctypes.c_float) for n in ("residual", "eps", "offset")] + [("type", ctypes.c_int)])


class I8Product(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("codes", "scales", "weights", "weight_scales", "bias", "y")]
                + [(n, ctypes.c_int64) for n in ("codes_row", "weights_row", "y_row", "rows", "N", "K")] + [("y_type", ctypes.c_int), ("gated", ctypes.c_int)])


def _device():
    torch = _b._torch or _b._load_torch()
    return torch.cuda.current_device() if torch.cuda.is_available() else -1


def _tensor(t, dtypes, shape, what, device):
    """t, a tensor on the current device whose last dimension is dense; None in the shape stands for any extent."""
    torch = _b._torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.dim() == len(shape)):
        raise SpqtError(f"{what}: need a CUDA tensor of {len(shape)} dimensions and dtype {' or '.join(str(d) for d in dtypes)}")
    if any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise SpqtError(f"{what}: shape {tuple(t.shape)} does not match {shape}")
    if t.device.index != device:
        raise SpqtError(f"{what}: on {t.device}, the current device is {device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise SpqtError(f"{what}: the last dimension has to be dense")
    return t


def _row(t):
    """Elements from one row to the next; of a single row the least that any check asks for."""
    return t.stride(0) if t.shape[0] > 1 else 0


def _types():
    torch = _b._torch or _b._load_torch()
    return torch, (torch.float16, torch.bfloat16)


def _type(t):
    return 1 if t.dtype == _b._torch.bfloat16 else 0


def _codes(codes, scales, shape, device, names=("codes", "scales")):
    torch = _b._torch
    c = _tensor(codes, (torch.int8,), shape, names[0], device)
    return c, _tensor(scales, (torch.float32,), (c.shape[0],), names[1], device)


def new_i8_codes(rows: int, K: int, device="cuda"):
    """An int8 tensor [rows, K] whose rows begin at multiples of 128 bytes, which is how products read them fastest; not initialized."""
    torch, _ = _types()
    if rows < 1 or K < 1:
        raise SpqtError("new_i8_codes: the extents are at least 1")
    width = -(-K // 128) * 128
    return torch.empty((rows, width), dtype=torch.int8, device=device)[:, :K]


def spqt_i8_quantize(x, codes, scales, stream=None) -> None:
    """Codes int8 [rows, K] and scales float32 [rows] of x [rows, K]."""
    if _b._fast is not None:
        rc = _b._fast.i8_quantize((_b._lib or lib()).at["spqt_i8_quantize"], x, codes, scales, stream)
        if rc is not None:
            return _check(rc)
    torch, halves = _types()
    device = _device()
    x = _tensor(x, halves, (None, None), "x", device)
    c, s = _codes(codes, scales, tuple(x.shape), device)
    _check(lib().spqt_i8_quantize(x.data_ptr(), _row(x), x.shape[0], x.shape[1], _type(x), c.data_ptr(), _row(c), s.data_ptr(), _b._stream_ptr(stream)))


def spqt_i8_read(codes, scales, out, stream=None) -> None:
    """out [rows, K] = code * scale."""
    if _b._fast is not None:
        rc = _b._fast.i8_read((_b._lib or lib()).at["spqt_i8_read"], codes, scales, out, stream)
        if rc is not None:
            return _check(rc)
    torch, halves = _types()
    device = _device()
    o = _tensor(out, halves, (None, None), "out", device)
    c, s = _codes(codes, scales, tuple(o.shape), device)
    _check(lib().spqt_i8_read(c.data_ptr(), _row(c), s.data_ptr(), o.shape[0], o.shape[1], _type(o), o.data_ptr(), _row(o), _b._stream_ptr(stream)))


def spqt_i8_norm(h, gain, out=None, codes=None, scales=None, block=None, block_gain=None, gate=None, residual: float = 1.0, eps: float = 1e-5,
                 offset: float = 0.0, h_out=None, stream=None) -> None:
    """The norms around a block, h [rows, K]: with block, h_out = residual * h + block, the block first normed with block_gain [K] and multiplied by gate ([K] or
    [rows, K]) if they are given; then out and / or codes and scales of that sum (of h, without a block) normed with gain [K].  Gains count from `offset` on.
    h_out may be h or block; out may be h or block."""
    if _b._fast is not None:
        rc = _b._fast.i8_norm((_b._lib or lib()).at["spqt_i8_norm"], h, gain, out, codes, scales, block, block_gain, gate, residual, eps, offset, h_out, stream)
        if rc is not None:
            return _check(rc)
    torch, halves = _types()
    device = _device()
    h = _tensor(h, halves, (None, None), "h", device)
    rows, K = h.shape
    shape, same = (rows, K), (h.dtype,)
    call = I8NormCall(h=h.data_ptr(), h_row=_row(h), rows=rows, K=K, residual=residual, eps=eps, offset=offset, type=_type(h),
                      gain=_tensor(gain, same, (K,), "gain", device).data_ptr())
    for name, t in (("block", block), ("h_out", h_out), ("out", out)):
        if t is not None:
            _tensor(t, same, shape, name, device)
            setattr(call, name, t.data_ptr())
            setattr(call, name + "_row", _row(t))
    if block_gain is not None:
        call.block_gain = _tensor(block_gain, same, (K,), "block_gain", device).data_ptr()
    if gate is not None:
        one = isinstance(gate, torch.Tensor) and gate.dim() == 1
        g = _tensor(gate, same, (K,) if one else shape, "gate", device)
        call.gate, call.gate_row = g.data_ptr(), 0 if one else _row(g)
    if codes is not None or scales is not None:
        c, s = _codes(codes, scales, shape, device)
        call.codes, call.codes_row, call.scales = c.data_ptr(), _row(c), s.data_ptr()
    _check(lib().spqt_i8_norm(ctypes.byref(call), _b._stream_ptr(stream)))


def spqt_i8_workspace_bytes(rows: int, N: int, K: int) -> int:
    """Bytes of a workspace for products of this size and of every smaller one."""
    out = ctypes.c_size_t()
    _check(lib().spqt_i8_workspace_bytes(rows, N, K, ctypes.byref(out)))
    return out.value


def new_i8_workspace(rows: int, N: int, K: int, device="cuda"):
    """A workspace tensor for spqt_i8_gemm of this size; calls of one stream may share one that is large enough for each of them, GEMVs may not."""
    torch, _ = _types()
    return torch.empty(max(256, spqt_i8_workspace_bytes(rows, N, K)), dtype=torch.uint8, device=device)


def spqt_i8_gemm(codes, scales, weights, weight_scales, y, bias=None, gated: bool = False, workspace=None, stream=None) -> None:
    """y [rows, N] float16, bfloat16 or float32 = (codes [rows, K] times weights int8 [N, K]) * scales [rows] * weight_scales [N] + bias float32 [N].
    gated: weights of N / 2 rows of a gate and, behind them, of an up projection; y [rows, N / 2] = silu(gate) * up.
    workspace (new_i8_workspace): lets K be divided where rows and channels alone do not fill the chip; None: y is the same, and the call may take longer."""
    if _b._fast is not None:
        rc = _b._fast.i8_gemm((_b._lib or lib()).at["spqt_i8_gemm"], codes, scales, weights, weight_scales, y, bias, gated, workspace, stream)
        if rc is not None:
            return _check(rc)
    torch, halves = _types()
    device = _device()
    c, s = _codes(codes, scales, (None, None), device)
    rows, K = c.shape
    w, ws = _codes(weights, weight_scales, (None, K), device, ("weights", "weight_scales"))
    N = w.shape[0]
    out = _tensor(y, halves + (torch.float32,), (rows, N // 2 if gated else N), "y", device)
    call = I8Product(codes=c.data_ptr(), scales=s.data_ptr(), weights=w.data_ptr(), weight_scales=ws.data_ptr(), y=out.data_ptr(), codes_row=_row(c),
                     weights_row=_row(w), y_row=_row(out), rows=rows, N=N, K=K, y_type=2 if out.dtype == torch.float32 else _type(out), gated=int(bool(gated)))
    if bias is not None:
        call.bias = _tensor(bias, (torch.float32,), (N,), "bias", device).data_ptr()
    space = None if workspace is None else _tensor(workspace, (torch.uint8,), (None,), "workspace", device)
    _check(lib().spqt_i8_gemm(ctypes.byref(call), None if space is None else space.data_ptr(), 0 if space is None else space.numel(), _b._stream_ptr(stream)))
