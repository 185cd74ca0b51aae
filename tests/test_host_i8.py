"""The entry points of the prompt side in 8-bit integers on the host: what the header declares is exported, and what is refused is refused before
anything is launched."""
import ctypes

import pytest

import paper_2511_04477_amd as spqt
from paper_2511_04477_amd.i8 import I8NormCall, I8Product
from test_host import declared_functions

EINVAL, ESHAPE, EALIGN, ESIZE = -1, -2, -3, -4
P = 1 << 20


def test_header_symbols_are_exported():
    names = [n for n in declared_functions("spqt_i8.h") if n.startswith("spqt_i8")]
    assert set(names) == set(spqt.I8_EXPORTS)
    for n in names:
        assert getattr(spqt.lib(), n) is not None


def quantize(x=P, x_row=64, rows=3, K=64, type=0, codes=2 * P, codes_row=64, scales=3 * P):
    return spqt.lib().spqt_i8_quantize(x, x_row, rows, K, type, codes, codes_row, scales, None)


def read(x=P, x_row=64, rows=3, K=64, type=0, codes=2 * P, codes_row=64, scales=3 * P):
    return spqt.lib().spqt_i8_read(codes, codes_row, scales, rows, K, type, x, x_row, None)


ROWS = [(dict(x=None), EINVAL), (dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(type=2), EINVAL), (dict(type=-1), EINVAL), (dict(x_row=-1), EINVAL),
        (dict(codes_row=-16), EINVAL), (dict(rows=0), ESHAPE), (dict(rows=-1), ESHAPE), (dict(rows=(1 << 24) + 1), ESHAPE), (dict(K=0), ESHAPE), (dict(K=131072), ESHAPE),
        (dict(x=P + 1), EALIGN), (dict(codes=2 * P + 8), EALIGN), (dict(codes_row=72), EALIGN), (dict(scales=3 * P + 2), EALIGN), (dict(x_row=(1 << 40) + 1), ESHAPE)]


@pytest.mark.parametrize("bad,status", ROWS)
def test_rows_that_are_refused(bad, status):
    assert quantize(**bad) == status
    assert read(**bad) == status


def test_rows_that_would_be_written_over_each_other_are_refused():
    assert quantize(codes_row=48) == EINVAL and read(x_row=63) == EINVAL
    assert quantize(K=65537, x_row=1 << 17, codes_row=1 << 17) == ESHAPE


def norm(**more):
    given = dict(h=P, block=2 * P, block_gain=3 * P, gate=4 * P, gain=5 * P, h_out=6 * P, out=7 * P, codes=8 * P, scales=9 * P, h_row=64, block_row=64, gate_row=64, h_out_row=64,
                 out_row=64, codes_row=64, rows=3, K=64, residual=1.0, eps=1e-5, offset=0.0, type=0)
    given.update(more)
    call = I8NormCall(**given)
    return spqt.lib().spqt_i8_norm(ctypes.byref(call), None)


@pytest.mark.parametrize("bad,status", [
    (dict(h=None), EINVAL), (dict(gain=None), EINVAL), (dict(type=2), EINVAL), (dict(block=None), EINVAL), (dict(h_out=None), EINVAL), (dict(block=None, h_out=None), EINVAL),
    (dict(block=None, h_out=None, gate=None), EINVAL), (dict(block=None, h_out=None, block_gain=None), EINVAL), (dict(codes=None), EINVAL), (dict(scales=None), EINVAL),
    (dict(block=None, block_gain=None, gate=None, h_out=None, out=None, codes=None, scales=None), EINVAL), (dict(out=6 * P), EINVAL),
    (dict(eps=0.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(eps=-1.0), EINVAL), (dict(residual=float("inf")), EINVAL),
    (dict(offset=float("nan")), EINVAL), (dict(rows=0), ESHAPE), (dict(rows=(1 << 24) + 1), ESHAPE), (dict(K=0), ESHAPE), (dict(K=65537), ESHAPE),
    (dict(h_row=-64), EINVAL), (dict(block_row=-64), EINVAL), (dict(gate_row=-64), EINVAL), (dict(h_out_row=63), EINVAL), (dict(out_row=0), EINVAL), (dict(codes_row=48), EINVAL),
    (dict(codes_row=72), EALIGN), (dict(codes=8 * P + 8), EALIGN), (dict(scales=9 * P + 2), EALIGN)] + [(dict([(n, P * 10 + 1)]), EALIGN) for n in
                                                                                                         ("h", "block", "block_gain", "gate", "gain", "h_out", "out")])
def test_norms_that_are_refused(bad, status):
    assert norm(**bad) == status


def test_a_norm_needs_its_call():
    assert spqt.lib().spqt_i8_norm(None, None) == EINVAL
    assert spqt.lib().spqt_i8_gemm(None, None, 0, None) == EINVAL


def product(workspace=None, size=0, **more):
    given = dict(codes=P, scales=2 * P, weights=3 * P, weight_scales=4 * P, bias=5 * P, y=6 * P, codes_row=64, weights_row=64, y_row=32, rows=3, N=32, K=64, y_type=0, gated=0)
    given.update(more)
    call = I8Product(**given)
    return spqt.lib().spqt_i8_gemm(ctypes.byref(call), workspace, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(weights=None), EINVAL), (dict(weight_scales=None), EINVAL), (dict(y=None), EINVAL), (dict(y_type=3), EINVAL),
    (dict(gated=2), EINVAL), (dict(codes_row=-16), EINVAL), (dict(weights_row=-16), EINVAL), (dict(y_row=31), EINVAL), (dict(y_row=15, gated=1), EINVAL), (dict(rows=0), ESHAPE),
    (dict(rows=(1 << 24) + 1), ESHAPE), (dict(N=0), ESHAPE), (dict(N=(1 << 24) + 1), ESHAPE), (dict(K=0), ESHAPE), (dict(K=131072), ESHAPE), (dict(N=33, gated=1), ESHAPE),
    (dict(codes=P + 8), EALIGN), (dict(weights=3 * P + 4), EALIGN), (dict(codes_row=72), EALIGN), (dict(weights_row=72), EALIGN), (dict(scales=2 * P + 2), EALIGN),
    (dict(weight_scales=4 * P + 1), EALIGN), (dict(bias=5 * P + 2), EALIGN), (dict(y=6 * P + 1), EALIGN), (dict(y=6 * P + 2, y_type=2), EALIGN),
    (dict(workspace=P + 128, size=1 << 30), EALIGN)])
def test_products_that_are_refused(bad, status):
    assert product(**bad) == status


def test_workspace_sizes():
    size = spqt.spqt_i8_workspace_bytes
    out = ctypes.c_size_t()
    L = spqt.lib()
    assert L.spqt_i8_workspace_bytes(1, 1, 1, None) == EINVAL
    for bad in [(0, 1, 1), (1, 0, 1), (1, 1, 0), ((1 << 24) + 1, 1, 1), (1, (1 << 24) + 1, 1), (1, 1, 131072)]:
        assert L.spqt_i8_workspace_bytes(*bad, ctypes.byref(out)) == ESHAPE
        with pytest.raises(spqt.SpqtError):
            size(*bad)
    for rows in (1, 16, 40, 64, 100, 250, 512, 4000):
        for N in (1, 512, 4096, 28672):
            for K in (16, 1000, 4096, 28672):
                need = size(rows, N, K)
                assert 0 <= need <= 1 << 28
                if need:                          # a workspace that is too small is refused, none is not asked for
                    assert product(workspace=P, size=need - 1, rows=rows, N=N, K=K, codes_row=K + 16 - K % 16, weights_row=K + 16 - K % 16, y_row=N) == ESIZE


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x, c, s = torch.zeros((2, 32), dtype=torch.float16), torch.zeros((2, 32), dtype=torch.int8), torch.zeros(2)
    for call in (lambda: spqt.spqt_i8_quantize(x, c, s), lambda: spqt.spqt_i8_read(c, s, x), lambda: spqt.spqt_i8_norm(x, x[0], out=x), lambda: spqt.spqt_i8_gemm(c, s, c, s, x),
                 lambda: spqt.spqt_i8_quantize(None, c, s), lambda: spqt.spqt_i8_gemm(c, s, None, s, x), lambda: spqt.new_i8_codes(0, 4), lambda: spqt.new_i8_codes(4, 0)):
        with pytest.raises(spqt.SpqtError):
            call()


def test_codes_that_the_binding_makes_begin_at_multiples_of_128_bytes():
    for rows, K in ((2, 1), (3, 16), (5, 17), (4, 4096), (2, 5003), (2, 8192)):
        c = spqt.new_i8_codes(rows, K, device="cpu")
        assert tuple(c.shape) == (rows, K) and c.stride(1) == 1 and c.stride(0) % 128 == 0 and c.stride(0) >= K
