"""The prompt side in 8-bit integers on the GPU: codes and what they stand for bit for bit, norms and products against 64 bits."""
import math

import pytest
import torch

from oracle import i8 as oracle

pytestmark = pytest.mark.gpu

TYPES = ["float16", "bfloat16"]


@pytest.fixture(scope="module")
def gpu():
    import paper_2511_04477_amd as spqt
    assert torch.cuda.is_available()
    assert spqt.lib()
    return spqt


def same(a, b):
    """Bit for bit, any NaN being as good as any other."""
    return a.dtype == b.dtype and torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0)) and torch.equal(a.isnan(), b.isnan())


def guarded(rows, width, pitch, dtype, at=0, fill=77):
    """A tensor [rows, width] inside a larger one that is filled with something; (view, whole)."""
    whole = torch.full((rows + 2, pitch), fill, dtype=dtype, device="cuda")
    return whole[1 : rows + 1, at : at + width], whole


def untouched(view, whole, fill=77):
    """Whether everything around the view is as it was."""
    copy = whole.clone()
    row, at = divmod(view.storage_offset() - whole.storage_offset(), whole.shape[1])
    copy[row : row + view.shape[0], at : at + view.shape[1]] = fill
    return bool((copy == fill).all())


def codes_like(rows, K, seed=0, more=0):
    """Any codes, in rows with anything behind them."""
    gen = torch.Generator().manual_seed(seed)
    whole = torch.randint(-128, 128, (rows, -(-K // 16) * 16 + more), generator=gen, dtype=torch.int32).to(torch.int8).cuda()
    return whole[:, :K]


def rounded_to(y, want, off, dtype):
    """|y - want| within off and half a step of y's type."""
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    return bool(((y.double().cpu() - want).abs() <= off + (want.abs() + off) * oracle.half_step(dtype) + tiny / 2).all())


# ---------------------------------------------------------------------------- codes

WIDTHS = [1, 7, 8, 9, 511, 512, 513, 2047, 2048, 2049, 4096, 4097, 5003, 8192, 8193, 16384, 16390, 32768, 32777, 65535, 65536]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", WIDTHS)
def test_codes(gpu, K, dtype):
    dtype = getattr(torch, dtype)
    rows = 9 if K < 10000 else 3
    gen = torch.Generator().manual_seed(K)
    x = (torch.randn((rows, K), generator=gen) * torch.exp(2 * torch.randn((rows, 1), generator=gen))).to(dtype)
    for at, pitch in ((0, K), (1, K + 3), (8, K + 24)):
        wide = torch.full((rows, pitch), float("nan"), dtype=dtype)
        wide[:, at : at + K] = x
        given = wide.cuda()[:, at : at + K]
        codes, whole = guarded(rows, K, -(-K // 16) * 16 + 32, torch.int8, 16)
        scales = torch.zeros(rows, device="cuda")
        gpu.spqt_i8_quantize(given, codes, scales)
        want, want_scales = oracle.quantize(x)
        assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want) and untouched(codes, whole)
        out, whole_out = guarded(rows, K, K + 5, dtype, 3)
        gpu.spqt_i8_read(codes, scales, out)
        assert same(out.cpu(), oracle.read(want, want_scales, dtype)) and untouched(out, whole_out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 40, 700, 3000, 9001])
def test_rows_that_are_no_ordinary_numbers(gpu, K, dtype):
    dtype = getattr(torch, dtype)
    info = torch.finfo(dtype)
    x = torch.randn((10, K), generator=torch.Generator().manual_seed(1)).to(dtype)
    x[0] = 0
    x[1] = -0.0
    x[2, K // 2] = math.inf
    x[3, K - 1] = math.nan
    x[4] = info.max
    x[5, 0] = -info.max
    x[6] = info.smallest_normal * info.eps           # the least number there is
    x[7] = x[7] * info.smallest_normal
    x[8, K - 1] = -math.inf
    x[9] = x[9].abs().max() / 2                      # half of the largest: half way between two codes
    x[9, 0] = x[9, 0] * 2
    codes, scales = gpu.new_i8_codes(10, K), torch.zeros(10, device="cuda")
    gpu.spqt_i8_quantize(x.cuda(), codes, scales)
    want, want_scales = oracle.quantize(x)
    assert same(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want)
    assert scales[[2, 3, 8]].isnan().all() and not scales[[0, 1, 4, 5, 6, 7, 9]].isnan().any()
    out = torch.zeros((10, K), dtype=dtype, device="cuda")
    gpu.spqt_i8_read(codes, scales, out)
    assert same(out.cpu(), oracle.read(want, want_scales, dtype))
    assert bool(torch.isfinite(out[4:6]).all())      # 127 scales of the largest number may be more than it
    # what such a row makes of a product
    w = codes_like(33, K, 5)
    y = torch.zeros((10, 33), device="cuda")
    gpu.spqt_i8_gemm(codes, scales, w, torch.ones(33, device="cuda"), y)
    assert y[[2, 3, 8]].isnan().all() and torch.isfinite(y[[0, 1, 6, 7, 9]]).all() and (y[:2] == 0).all()


@pytest.mark.parametrize("rows,K", [(1, 300), (4097, 40), (70000, 8), (2049, 2000)])
def test_codes_of_many_rows(gpu, rows, K):
    x = torch.randn((rows, K), generator=torch.Generator().manual_seed(3)).half()
    codes, scales = gpu.new_i8_codes(rows, K), torch.zeros(rows, device="cuda")
    gpu.spqt_i8_quantize(x.cuda(), codes, scales)
    top = x.float().abs().amax(dim=1, keepdim=True)
    assert torch.equal(codes.cpu(), torch.round(x.float() * (torch.tensor(127.0) / top)).to(torch.int8)) and torch.equal(scales.cpu(), top[:, 0] / 127.0)
    out = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
    gpu.spqt_i8_read(codes, scales, out)
    assert same(out.cpu(), oracle.read(codes.cpu(), scales.cpu(), torch.float16))


@pytest.mark.parametrize("K", [131071, 70000])
def test_the_widest_rows_are_read_back(gpu, K):
    codes, scales = codes_like(2, K), torch.tensor([0.5, 3.0], device="cuda")
    out = torch.zeros((2, K), dtype=torch.bfloat16, device="cuda")
    gpu.spqt_i8_read(codes, scales, out)
    assert same(out.cpu(), oracle.read(codes.cpu(), scales.cpu(), torch.bfloat16))


# ---------------------------------------------------------------------------- norms

FORMS = [dict(block=False), dict(), dict(block_gain=True), dict(gate="channel"), dict(gate="row", residual=0.75),
         dict(block_gain=True, gate="channel", offset=1.0), dict(block_gain=True, gate="row", residual=-0.5, eps=1e-3)]


def norm_inputs(rows, K, dtype, form, seed=0, pitch=None):
    gen = torch.Generator().manual_seed(seed + K)
    offset = form.get("offset", 0.0)

    def normal(*shape):
        return torch.randn(shape, generator=gen)

    given = {"h": (normal(rows, K) * torch.exp(0.7 * normal(K))).to(dtype), "gain": (1 - offset + 0.3 * normal(K)).to(dtype)}
    if form.get("block", True):
        given["block"] = (normal(rows, K) * 2).to(dtype)
        if form.get("block_gain"):
            given["block_gain"] = (1 - offset + 0.3 * normal(K)).to(dtype)
        if form.get("gate"):
            given["gate"] = normal(*((K,) if form["gate"] == "channel" else (rows, K))).to(dtype)
    return given, {n: form[n] for n in ("residual", "eps", "offset") if n in form}


def check_norm(gpu, given, more, outputs, dtype):
    s, x, off, far = oracle.norm(**{n: t.double() for n, t in given.items()}, **more)
    if "h_out" in outputs:
        assert rounded_to(outputs["h_out"], s, off, dtype)
    if "out" in outputs:
        assert rounded_to(outputs["out"], x, far, dtype)
    if "codes" in outputs:
        scales, codes = outputs["scales"].double().cpu(), outputs["codes"].double().cpu()
        top = x.abs().max(dim=1)[0]
        assert bool(((scales * 127 - top).abs() <= far.max(dim=1)[0] + 2 * oracle.U * top).all())
        # half a scale, what x is off by, and two roundings of up to 127
        assert bool(((codes * scales[:, None] - x).abs() <= 0.5 * scales[:, None] + far + (x.abs() + scales[:, None]) * 4 * oracle.U).all())
        assert int(outputs["codes"].abs().max()) == 127


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f"{k}={v}" for k, v in f.items()) or "join")
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 8, 75, 512, 1000, 2048, 2111, 4096, 8192, 8200, 16384, 20001, 32768, 40003, 65536])
def test_norm(gpu, K, dtype, form):
    dtype = getattr(torch, dtype)
    rows = 5 if K < 10000 else 2
    given, more = norm_inputs(rows, K, dtype, form)
    on = {n: t.cuda() for n, t in given.items()}
    outputs, wholes = {}, {}
    for n, at in (("h_out", 1), ("out", 8)):
        if n == "out" or "block" in given:
            outputs[n], wholes[n] = guarded(rows, K, K + 17, dtype, at)
    outputs["codes"], wholes["codes"] = guarded(rows, K, -(-K // 16) * 16 + 16, torch.int8, 16)
    outputs["scales"] = torch.zeros(rows, device="cuda")
    gpu.spqt_i8_norm(**on, **more, **outputs)
    check_norm(gpu, given, more, outputs, dtype)
    assert all(untouched(outputs[n], wholes[n]) for n in wholes)
    # one output alone is the same
    alone = {n: torch.zeros_like(outputs[n]) for n in outputs if n == "h_out"}
    out = torch.zeros((rows, K), dtype=dtype, device="cuda")
    gpu.spqt_i8_norm(**on, **more, out=out, **alone)
    assert same(out, outputs["out"])
    codes, scales = gpu.new_i8_codes(rows, K), torch.zeros(rows, device="cuda")
    gpu.spqt_i8_norm(**on, **more, codes=codes, scales=scales, **alone)
    assert torch.equal(codes, outputs["codes"]) and torch.equal(scales, outputs["scales"])


@pytest.mark.parametrize("K", [64, 2500, 8192])
def test_norm_in_place_and_of_slices(gpu, K):
    dtype = torch.bfloat16
    given, more = norm_inputs(7, K, dtype, dict(block_gain=True, gate="row"))
    on = {n: t.cuda() for n, t in given.items()}
    h_out, out = (torch.zeros((7, K), dtype=dtype, device="cuda") for _ in range(2))
    gpu.spqt_i8_norm(**on, **more, h_out=h_out, out=out)
    for first, second in (("h", "block"), ("block", "h"), ("h", None), ("block", None)):
        now = {n: t.clone() for n, t in on.items()}
        other = torch.zeros((7, K), dtype=dtype, device="cuda") if second is None else now[second]
        gpu.spqt_i8_norm(**now, **more, h_out=now[first], out=other)
        assert same(now[first], h_out) and same(other, out)
    # slices of wider tensors, at odd places; one row of a gate or of h for all
    wide = torch.randn((7, 3 * K + 9), generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
    parts = {"h": wide[:, 1 : K + 1], "block": wide[:, K + 3 : 2 * K + 3], "gate": wide[:, 2 * K + 8 : 3 * K + 8]}
    gpu.spqt_i8_norm(gain=on["gain"], h_out=h_out, out=out, **parts)
    check_norm(gpu, dict({n: t.cpu() for n, t in parts.items()}, gain=given["gain"]), {}, {"h_out": h_out, "out": out}, dtype)
    parts = {"h": on["h"][:1].expand(7, K), "block": on["block"], "gate": on["gate"][:1].expand(7, K)}
    gpu.spqt_i8_norm(gain=on["gain"], h_out=h_out, out=out, **parts)
    check_norm(gpu, dict({n: t.cpu() for n, t in parts.items()}, gain=given["gain"]), {}, {"h_out": h_out, "out": out}, dtype)


@pytest.mark.parametrize("K", [5, 3000])
def test_norm_of_rows_that_are_no_ordinary_numbers(gpu, K):
    dtype = torch.bfloat16
    h = torch.randn((6, K), generator=torch.Generator().manual_seed(2)).to(dtype)
    h[0] = 0
    h[1] = h[1] * 1e30                               # squares leave fp32
    h[2] = h[2] * 1e-30
    h[3, K - 1] = math.nan
    h[4, 0] = math.inf
    gain = torch.ones(K, dtype=dtype)
    out, codes, scales = torch.zeros((6, K), dtype=dtype, device="cuda"), gpu.new_i8_codes(6, K), torch.zeros(6, device="cuda")
    gpu.spqt_i8_norm(h.cuda(), gain.cuda(), out=out, codes=codes, scales=scales)
    keep = [0, 1, 2, 5]
    _, x, _, far = oracle.norm(h[keep].double(), gain.double())
    assert rounded_to(out[keep], x, far + 1e-38, dtype)
    assert bool(out[3].isnan().all()) and bool(scales[3:5].isnan().all()) and bool((codes[3:5] == 0).all())
    assert bool((codes[0] == 0).all()) and torch.isfinite(scales[keep]).all()


@pytest.mark.parametrize("K", [7, 4096, 20000, 65536])
def test_norm_of_the_largest_numbers(gpu, K):
    dtype = torch.bfloat16
    h = torch.full((3, K), torch.finfo(dtype).max, dtype=dtype)
    h[0, 1::2] *= -1
    h[1] *= 2.0**-71                                 # whose squares are numbers of fp32 and whose sum is one or not, by K
    h[2, K // 2 :] = 1.0
    gain = torch.randn(K, generator=torch.Generator().manual_seed(K)).to(dtype)
    out, codes, scales = torch.zeros((3, K), dtype=dtype, device="cuda"), gpu.new_i8_codes(3, K), torch.zeros(3, device="cuda")
    gpu.spqt_i8_norm(h.cuda(), gain.cuda(), out=out, codes=codes, scales=scales)
    _, x, _, far = oracle.norm(h.double(), gain.double())
    far = far + x.abs() * 2.0**-21                   # 1 / 2^128 is a subnormal number of 22 bits
    assert rounded_to(out, x, far + 1e-38, dtype)
    top = x.abs().max(dim=1)[0]
    assert bool(((scales.double().cpu() * 127 - top).abs() <= far.max(dim=1)[0] + 2 * oracle.U * top).all())


@pytest.mark.parametrize("rows,K", [(5001, 24), (3001, 1000), (1500, 4096), (300, 8192), (333, 5003), (257, 14336), (261, 9007), (258, 20000)])
def test_norm_of_many_rows(gpu, rows, K):
    given, more = norm_inputs(rows, K, torch.float16, dict(block_gain=True, gate="channel"))
    on = {n: t.cuda() for n, t in given.items()}
    outputs = {"h_out": torch.zeros_like(on["h"]), "out": torch.zeros_like(on["h"]), "codes": gpu.new_i8_codes(rows, K), "scales": torch.zeros(rows, device="cuda")}
    gpu.spqt_i8_norm(**on, **outputs)
    check_norm(gpu, given, more, outputs, torch.float16)
    # a row does not depend on the others
    for r in (0, rows // 2, rows - 1):
        one = torch.zeros((1, K), dtype=torch.float16, device="cuda")
        gpu.spqt_i8_norm(on["h"][r : r + 1], on["gain"], block=on["block"][r : r + 1], block_gain=on["block_gain"], gate=on["gate"], h_out=torch.zeros_like(one), out=one)
        assert same(one[0], outputs["out"][r])
    # in place
    gpu.spqt_i8_norm(**on, h_out=on["h"], out=on["block"])
    assert same(on["h"], outputs["h_out"]) and same(on["block"], outputs["out"])


# ------------------------------------------------------------------------- products

SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 129), (3, 70, 16), (5, 33, 1000), (16, 64, 4096), (17, 100, 5003), (33, 300, 640), (40, 1000, 2100), (64, 48, 9000),
          (65, 130, 500), (100, 515, 300), (129, 257, 1024), (250, 600, 3500), (256, 256, 128), (257, 511, 777), (300, 520, 2000), (513, 1030, 400), (1100, 700, 192)]


def product_inputs(rows, N, K, seed=0, bias=False):
    gen = torch.Generator().manual_seed(seed + 31 * rows + 7 * N + K)
    codes, weights = codes_like(rows, K, seed + 1, 16 * (seed % 3)), codes_like(N, K, seed + 2, 16 * (seed % 2))
    scales = torch.exp(torch.randn(rows, generator=gen)) * 0.01
    weight_scales = torch.exp(0.3 * torch.randn(N, generator=gen)) * (0.02 / math.sqrt(K))
    return codes, scales.cuda(), weights, weight_scales.cuda(), torch.randn(N, generator=gen).cuda() if bias else None


def check_product(gpu, inputs, dtype, gated=False, space=None, pitch=3, at=1):
    codes, scales, weights, weight_scales, bias = inputs
    rows, outputs = codes.shape[0], weights.shape[0] // (2 if gated else 1)
    y, whole = guarded(rows, outputs, outputs + pitch, dtype, at)
    gpu.spqt_i8_gemm(codes, scales, weights, weight_scales, y, bias=bias, gated=gated, workspace=space)
    want, off = oracle.product(codes.cpu(), scales.cpu(), weights.cpu(), weight_scales.cpu(), None if bias is None else bias.cpu(), gated)
    assert rounded_to(y, want, off, dtype) and untouched(y, whole)
    return y


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,N,K", SHAPES)
def test_products(gpu, rows, N, K, dtype):
    dtype = getattr(torch, dtype)
    seed = (rows + N) % 5
    inputs = product_inputs(rows, N, K, seed, bias=seed % 2 == 1)
    y = check_product(gpu, inputs, dtype)
    space = gpu.new_i8_workspace(rows, N, K)
    space.fill_(255)                                  # needs no preparation
    assert same(check_product(gpu, inputs, dtype, space=space), y)
    assert same(check_product(gpu, inputs, dtype, space=space, pitch=(8 - N) % 8, at=0), y)
    if N % 2 == 0:
        g = check_product(gpu, inputs, dtype, gated=True)
        assert same(check_product(gpu, inputs, dtype, gated=True, space=space, pitch=(8 - N // 2) % 8, at=0), g)


# Sizes that different tiles and numbers of parts are taken for, with edges in every dimension.
LARGE = [(771, 14331, 4101), (1021, 8183, 28672), (1500, 5118, 5131), (16, 8191, 28672), (7, 16390, 17000), (26, 1682, 7051), (61, 4090, 4100), (300, 521, 2000), (509, 10222, 8192), (1019, 4090, 4109), (250, 4094, 14336), (40, 8190, 28672), (127, 2050, 20000),
         (4001, 3070, 1000), (8000, 598, 400), (2047, 2050, 130), (65, 128, 131071)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows,N,K", LARGE)
def test_large_products(gpu, rows, N, K, dtype):
    """Bit for bit what sixteen rows at a time give, and a few rows of that against 64 bits."""
    dtype = getattr(torch, dtype)
    codes, scales, weights, weight_scales, _ = product_inputs(rows, N, K, 3)
    space = gpu.new_i8_workspace(rows, N, K)
    space.fill_(255)
    for gated in (False, True):
        if gated and N % 2:
            weights, weight_scales, N = weights[:-1], weight_scales[:-1], N - 1
        outputs = N // 2 if gated else N
        want = torch.zeros((rows, outputs), dtype=dtype, device="cuda")
        for r in range(0, rows, 16):
            gpu.spqt_i8_gemm(codes[r : r + 16], scales[r : r + 16], weights, weight_scales, want[r : r + 16], gated=gated)
        for given in (None, space):
            y, whole = guarded(rows, outputs, outputs + 2, dtype, 1)
            gpu.spqt_i8_gemm(codes, scales, weights, weight_scales, y, gated=gated, workspace=given)
            assert same(y, want) and untouched(y, whole)
        some = [0, 1, rows // 2, rows - 1]
        exact, off = oracle.product(codes[some].cpu(), scales[some].cpu(), weights.cpu(), weight_scales.cpu(), gated=gated)
        assert rounded_to(want[some], exact, off, dtype)


def test_a_workspace_for_more_serves_less(gpu):
    space = gpu.new_i8_workspace(600, 4096, 9000)
    for rows, N, K in ((600, 4096, 9000), (17, 40, 300), (250, 4000, 8999), (1, 4096, 9000), (600, 4096, 127)):
        inputs = product_inputs(rows, N, K)
        y, z = (torch.zeros((rows, N), device="cuda") for _ in range(2))
        gpu.spqt_i8_gemm(*inputs[:4], y, workspace=space)
        gpu.spqt_i8_gemm(*inputs[:4], z)
        assert same(y, z)


def test_a_gemv_on_a_products_workspace_gives_no_numbers(gpu):
    """A product leaves sums where a GEMV relies on zeros: such a GEMV yields NaN until the workspace is prepared again."""
    import numpy as np
    from workloads import make_case, quantile_threshold
    case = make_case(1, "w")
    M, K = case["M"], case["K"]
    packed, x = torch.from_numpy(gpu.spqt_pack(case["q_rowmajor"], case["scales"])).cuda(), torch.from_numpy(case["x"][0]).cuda()
    space = gpu.new_i8_workspace(250, 4096, 14336)
    assert space.numel() >= gpu.spqt_workspace_bytes(M, K)
    gpu.spqt_workspace_init(space)
    inputs = product_inputs(250, 4096, 14336)
    y = torch.zeros((250, 4096), device="cuda")
    gpu.spqt_i8_gemm(*inputs[:4], y, workspace=space)
    out = torch.zeros(M, device="cuda")
    gpu.spqt_gemv_fused(packed, M, K, x, quantile_threshold(case["x"], 0.5), out, space)
    assert bool(out.isnan().any())
    gpu.spqt_workspace_init(space)
    gpu.spqt_gemv_fused(packed, M, K, x, quantile_threshold(case["x"], 0.5), out, space)
    assert bool(torch.isfinite(out).all()) and np.isfinite(float(out.abs().max()))


@pytest.mark.parametrize("rows,N", [(1, 20), (20, 40), (130, 140), (300, 300), (513, 1000)])
def test_the_longest_sums_are_exact(gpu, rows, N):
    K = 131071
    codes = torch.full((rows, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    weights = torch.full((N, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    codes[:, 5] = torch.arange(rows, device="cuda") % 100
    one = torch.ones(max(rows, N), device="cuda")
    for space in (None, gpu.new_i8_workspace(rows, N, K)):
        y = torch.zeros((rows, N), device="cuda")
        gpu.spqt_i8_gemm(codes, one[:rows], weights, one[:N], y, workspace=space)
        want = (131070 * 16384 - 128 * (torch.arange(rows) % 100))[:, None].expand(rows, N).float()
        assert torch.equal(y.cpu(), want)


def test_scales_that_are_no_ordinary_numbers(gpu):
    inputs = list(product_inputs(40, 50, 300))
    inputs[1][3], inputs[1][7], inputs[1][9] = math.nan, 0.0, -2.0
    inputs[3][11], inputs[3][12] = math.nan, math.inf
    y = torch.zeros((40, 50), device="cuda")
    gpu.spqt_i8_gemm(*inputs[:4], y)
    assert y[3].isnan().all() and y[:, 11].isnan().all()
    inputs[1][3] = 1.0
    inputs[3][11:13] = 1.0
    z = check_product(gpu, inputs, torch.float32)
    keep = [r for r in range(40) if r != 3]
    cols = [n for n in range(50) if n not in (11, 12)]
    assert same(y[keep][:, cols], z[keep][:, cols]) and (z[7] == 0).all()


def test_products_over_32_bits_of_places(gpu):
    """Rows so far apart that their places pass 2^31."""
    K, pitch = 64, 1 << 26
    whole = torch.zeros(40 * pitch, dtype=torch.int8, device="cuda")
    codes = whole.view(40, pitch)[:, 256 : 256 + K]
    weights = whole.view(40, pitch)[:, 1024 : 1024 + K]
    given = product_inputs(40, 40, K)
    codes.copy_(given[0])
    weights.copy_(given[2])
    check_product(gpu, (codes, given[1], weights, given[3], None), torch.float16)
    x = whole[: 36 * pitch].view(torch.float16).view(18, pitch)[:, 4096 : 4096 + K]
    x.copy_(torch.randn((18, K), generator=torch.Generator().manual_seed(1)))
    out_codes, scales = whole.view(40, pitch)[:18, 65536 : 65536 + K], torch.zeros(18, device="cuda")
    gpu.spqt_i8_quantize(x, out_codes, scales)
    want, want_scales = oracle.quantize(x.cpu())
    assert torch.equal(out_codes.cpu(), want) and torch.equal(scales.cpu(), want_scales)


# ------------------------------------------------------------------------- together

class PromptLayer:
    """A decoder layer's prompt on these calls and the 8-bit cache, and the same in 64 bits from the codes that each step was given."""

    def __init__(self, spqt, hidden, heads, kv_heads, dim, inner, dtype, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.spqt, self.heads, self.kv_heads, self.dim, self.dtype, self.hidden = spqt, heads, kv_heads, dim, dtype, hidden
        self.weights = {}
        for name, (N, K) in {"qkv": ((heads + 2 * kv_heads) * dim, hidden), "o": (hidden, heads * dim), "gate_up": (2 * inner, hidden), "down": (hidden, inner)}.items():
            w = (torch.randn((N, K), generator=gen) / math.sqrt(K)).to(dtype).cuda()
            codes, scales = spqt.new_i8_codes(N, K), torch.zeros(N, device="cuda")
            spqt.spqt_i8_quantize(w, codes, scales)
            self.weights[name] = (codes, scales)
        self.gains = {n: (1 + 0.2 * torch.randn(hidden, generator=gen)).to(dtype).cuda() for n in ("first", "after", "second", "last")}
        self.space = spqt.new_i8_workspace(512, 2 * inner, max(hidden, inner))
        self.kv = spqt.new_kv_cache(16, kv_heads, dim, 1, dtype)
        self.table = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 16)
        self.attention_space = spqt.new_kv_workspace(1, 512, heads, kv_heads, dim, 16)
        self.seen = []

    def product(self, name, codes, scales, gated=False):
        w, ws = self.weights[name]
        y = torch.empty((codes.shape[0], w.shape[0] // (2 if gated else 1)), dtype=self.dtype, device="cuda")
        self.spqt.spqt_i8_gemm(codes, scales, w, ws, y, gated=gated, workspace=self.space)
        self.seen.append((name, codes, scales, y, gated))
        return y

    def codes(self, rows, K):
        return self.spqt.new_i8_codes(rows, K), torch.empty(rows, device="cuda")

    def __call__(self, h, lengths):
        """h [rows, hidden], in place; what the next layer's first product is given comes back."""
        spqt, rows = self.spqt, h.shape[0]
        self.seen = []
        a = self.codes(rows, self.hidden)
        spqt.spqt_i8_norm(h, self.gains["first"], codes=a[0], scales=a[1])
        qkv = self.product("qkv", *a).view(1, rows, -1, self.dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=2)
        spqt.spqt_kv_append(*self.kv[:3], self.table, lengths, k, v)
        out = torch.empty((1, rows, self.heads, self.dim), dtype=self.dtype, device="cuda")
        spqt.spqt_kv_attention(*self.kv[:2], self.table, lengths, q, out, self.attention_space)
        b = self.codes(rows, self.heads * self.dim)
        spqt.spqt_i8_quantize(out.view(rows, -1), *b)
        block = self.product("o", *b)
        c = self.codes(rows, self.hidden)
        spqt.spqt_i8_norm(h, self.gains["second"], block=block, block_gain=self.gains["after"], h_out=h, codes=c[0], scales=c[1])
        inner = self.product("gate_up", *c, gated=True)
        d = self.codes(rows, inner.shape[1])
        spqt.spqt_i8_quantize(inner, *d)
        block = self.product("down", *d)
        last = torch.empty_like(h)
        spqt.spqt_i8_norm(h, self.gains["last"], block=block, residual=0.5, h_out=h, out=last)
        return last


@pytest.mark.parametrize("dtype", TYPES)
def test_a_prompt_through_a_layer(gpu, dtype):
    dtype = getattr(torch, dtype)
    layer = PromptLayer(gpu, 320, 5, 1, 64, 700, dtype)
    gen = torch.Generator().manual_seed(4)
    done = 0
    for rows in (300, 1, 37, 4):                      # a prompt, a token, another prompt, drafts
        h = torch.randn((rows, 320), generator=gen).to(dtype).cuda()
        done += rows
        lengths = torch.tensor([done], dtype=torch.int32, device="cuda")
        before = h.clone()
        last = layer(h, lengths)
        assert [n for n, *_ in layer.seen] == ["qkv", "o", "gate_up", "down"] and not same(h, before)
        for name, codes, scales, y, gated in layer.seen:
            w, ws = layer.weights[name]
            want, off = oracle.product(codes.cpu(), scales.cpu(), w.cpu(), ws.cpu(), gated=gated)
            assert rounded_to(y, want, off, dtype)
        assert torch.isfinite(last.float()).all()


def test_replays_of_a_graph_and_other_streams(gpu):
    """The layer in a graph: each replay, with other inputs and eager work in between, as the eager call."""
    layer, other = PromptLayer(gpu, 256, 4, 2, 64, 500, torch.float16), PromptLayer(gpu, 256, 4, 2, 64, 500, torch.float16)
    gen = torch.Generator().manual_seed(5)
    h, lengths = torch.zeros((70, 256), dtype=torch.float16, device="cuda"), torch.tensor([70], dtype=torch.int32, device="cuda")
    inputs = [torch.randn((70, 256), generator=gen).half().cuda() for _ in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h.copy_(inputs[0])
        layer(h, lengths)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            last = layer(h, lengths)
    torch.cuda.current_stream().wait_stream(side)
    for x in inputs + inputs[:2]:
        eager = x.clone()
        want = other(eager, lengths)
        torch.cuda.synchronize()
        h.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert same(last, want) and same(h, eager)
    with torch.cuda.stream(side):                     # a stream that is given
        side.wait_stream(torch.cuda.default_stream())
        inputs5 = product_inputs(50, 60, 700)
        y, z = (torch.zeros((50, 60), device="cuda") for _ in range(2))
        gpu.spqt_i8_gemm(*inputs5[:4], y)
    side.synchronize()
    gpu.spqt_i8_gemm(*inputs5[:4], z, stream=side)
    side.synchronize()
    assert same(y, z)


@pytest.mark.parametrize("quick", [True, False])
def test_calls_that_are_refused(gpu, monkeypatch, quick):
    from paper_2511_04477_amd import binding
    if not quick:
        monkeypatch.setattr(binding, "_fast", None)
    x, codes, scales = torch.zeros((4, 64), dtype=torch.float16, device="cuda"), gpu.new_i8_codes(4, 64), torch.zeros(4, device="cuda")
    w, ws, y = gpu.new_i8_codes(6, 64), torch.zeros(6, device="cuda"), torch.zeros((4, 6), device="cuda")
    gain = x[0].clone()
    bad = [lambda: gpu.spqt_i8_quantize(x.float(), codes, scales), lambda: gpu.spqt_i8_quantize(x, codes[:3], scales), lambda: gpu.spqt_i8_quantize(x, codes, scales[:3]),
           lambda: gpu.spqt_i8_quantize(x.t(), codes, scales), lambda: gpu.spqt_i8_quantize(x, codes.view(torch.uint8), scales),
           lambda: gpu.spqt_i8_quantize(x[:, :60], torch.zeros((4, 60), dtype=torch.int8, device="cuda"), scales),
           lambda: gpu.spqt_i8_quantize(x.cpu(), codes, scales), lambda: gpu.spqt_i8_quantize(x, codes[:1].expand(4, 64), scales),
           lambda: gpu.spqt_i8_read(codes, scales, x[:, :32]), lambda: gpu.spqt_i8_read(codes, scales.half(), x), lambda: gpu.spqt_i8_read(codes, scales, x[:1].expand(4, 64)),
           lambda: gpu.spqt_i8_norm(x, gain), lambda: gpu.spqt_i8_norm(x, gain[:60], out=x), lambda: gpu.spqt_i8_norm(x, gain, out=x, h_out=x.clone()),
           lambda: gpu.spqt_i8_norm(x, gain, out=x, block=x), lambda: gpu.spqt_i8_norm(x, gain, block=x, h_out=x, out=x), lambda: gpu.spqt_i8_norm(x, gain, codes=codes),
           lambda: gpu.spqt_i8_norm(x, gain, scales=scales), lambda: gpu.spqt_i8_norm(x, gain, out=x, gate=gain), lambda: gpu.spqt_i8_norm(x, gain, out=x, block_gain=gain),
           lambda: gpu.spqt_i8_norm(x, gain, out=x, eps=0.0), lambda: gpu.spqt_i8_norm(x, gain, out=x, residual=math.nan), lambda: gpu.spqt_i8_norm(x, gain.bfloat16(), out=x),
           lambda: gpu.spqt_i8_norm(x, gain, block=x.clone(), h_out=x, out=x.clone(), gate=gain[:3]),
           lambda: gpu.spqt_i8_gemm(codes, scales, w, ws, y[:, :5]), lambda: gpu.spqt_i8_gemm(codes, scales, w[:, :48], ws, y), lambda: gpu.spqt_i8_gemm(codes, scales, w, ws[:5], y),
           lambda: gpu.spqt_i8_gemm(codes, scales, w[:5], ws[:5], y[:, :2], gated=True), lambda: gpu.spqt_i8_gemm(codes, scales, w, ws, y.double()),
           lambda: gpu.spqt_i8_gemm(codes, scales, w, ws, y, bias=ws.half()), lambda: gpu.spqt_i8_gemm(codes[:, 8:56], scales, w[:, 8:56], ws, y),
           lambda: gpu.spqt_i8_gemm(codes, scales, w, ws, y, workspace=torch.zeros(300, dtype=torch.uint8, device="cuda")[1:]),
           lambda: gpu.spqt_i8_gemm(codes[:0], scales[:0], w, ws, y[:0]), lambda: gpu.spqt_i8_quantize(x[:, :0], codes[:, :0], scales)]
    for i, call in enumerate(bad):
        with pytest.raises(gpu.SpqtError):
            call()
            print("not refused:", i)


def test_the_extension_module_gives_the_same(gpu, monkeypatch):
    """Calls through _fastcall and through the Python code: the same bits, and the module takes the plain ones itself, slices and all."""
    from paper_2511_04477_amd import binding
    fast, left = binding._fast, []
    assert fast is not None

    class Watched:
        def __getattr__(self, name):
            def go(*a):
                rc = getattr(fast, name)(*a)
                left.extend([name] if rc is None else [])
                return rc
            return go

    x = torch.randn((9, 700), generator=torch.Generator().manual_seed(1)).half().cuda()
    w, weight_scales = codes_like(50, 690, 2), torch.rand(50, device="cuda")

    def calls():
        codes, scales, back = gpu.new_i8_codes(9, 690), torch.zeros(9, device="cuda"), torch.zeros((9, 690), dtype=torch.float16, device="cuda")
        gpu.spqt_i8_quantize(x[:, 10:], codes, scales)
        gpu.spqt_i8_read(codes, scales, back)
        h_out, out = torch.zeros_like(back), torch.zeros_like(back)
        gpu.spqt_i8_norm(x[:, 5:695], x[0, :690], block=x[:, 10:], block_gain=x[1, 3:693], gate=x[:, 1:691], residual=0.5, offset=1.0, h_out=h_out, out=out, codes=codes, scales=scales)
        one = torch.zeros_like(back)
        gpu.spqt_i8_norm(x[:, 5:695], x[0, :690], block=x[:, 10:], gate=x[3, :690], h_out=h_out, out=one)
        found = [codes, scales, back, h_out, out, one]
        for dtype in (torch.float16, torch.bfloat16, torch.float32):
            for gated in (False, True):
                y = torch.zeros((9, 60), dtype=dtype, device="cuda")[:, : 25 if gated else 50]
                gpu.spqt_i8_gemm(codes, scales, w, weight_scales, y, bias=weight_scales, gated=gated, workspace=gpu.new_i8_workspace(9, 50, 690) if gated else None)
                found.append(y)
        return [t.clone() for t in found]

    monkeypatch.setattr(binding, "_fast", None)
    want = calls()
    monkeypatch.setattr(binding, "_fast", Watched())
    assert all(same(a, b) for a, b in zip(calls(), want)) and not left
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = calls()
    side.synchronize()
    assert all(same(a, b) for a, b in zip(again, want)) and not left
