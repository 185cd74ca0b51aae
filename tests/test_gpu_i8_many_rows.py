"""So many rows that a launch's workgroups go through them more than once: the same as in calls of fewer rows."""
import pytest
import torch

from i8_paths import MANY
from test_gpu_i8 import gpu, same  # noqa: F401
from test_gpu_i8_ways import by_steps, inputs_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back():
    """Tensors of tens of gigabytes are not kept for the tests that follow."""
    yield
    torch.cuda.empty_cache()


GROUPS = 1 << 20                                          # workgroups of a launch, at most


def windows(rows, K, dtype, apart=8):
    """[rows, K] whose rows are windows of one buffer, `apart` elements from each other: all different, in little memory."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    return torch.randn(rows * apart + K, generator=gen, device="cuda", dtype=dtype).as_strided((rows, K), (apart, 1))


# rows of up to 512, four of which share a workgroup, and of a workgroup's 256, 512 and 1024 threads
@pytest.mark.parametrize("K", [24, 520, 4100, 8200, 16400])
def test_codes_and_norms(gpu, K):  # noqa: F811
    rows = (4 if K <= 512 else 1) * GROUPS + 5001
    x = windows(rows, K, torch.float16)
    gain = windows(1, K, torch.float16)[0]
    few = 100000

    def quantize(x, codes, scales):
        gpu.spqt_i8_quantize(x, codes, scales)

    def norm(x, codes, scales):
        gpu.spqt_i8_norm(x, gain, block=x, block_gain=gain, h_out=h_out[: x.shape[0]], codes=codes, scales=scales)

    h_out = torch.empty((rows, K), dtype=torch.float16, device="cuda")
    codes, scales = gpu.new_i8_codes(rows, K), torch.zeros(rows, device="cuda")
    some, some_scales = gpu.new_i8_codes(few, K), torch.zeros(few, device="cuda")
    for call in (quantize, norm):
        codes.fill_(-128)
        scales.fill_(-1.0)
        call(x, codes, scales)
        for at in range(0, rows, few):
            n = min(few, rows - at)
            call(x[at : at + n], some[:n], some_scales[:n])
            assert torch.equal(codes[at : at + n], some[:n]) and torch.equal(scales[at : at + n], some_scales[:n]), at
    del h_out
    out = torch.full((rows, K), 7.0, dtype=torch.float16, device="cuda")
    gpu.spqt_i8_norm(x, gain, out=out)
    back = torch.full((rows, K), 7.0, dtype=torch.float16, device="cuda")
    gpu.spqt_i8_read(codes, scales, back)
    for at in range(0, rows, few):
        n = min(few, rows - at)
        part = torch.empty((n, K), dtype=torch.float16, device="cuda")
        gpu.spqt_i8_norm(x[at : at + n], gain, out=part)
        assert same(out[at : at + n], part), at
        gpu.spqt_i8_read(codes[at : at + n], scales[at : at + n], part)
        assert same(back[at : at + n], part), at


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,N,K,tile", MANY)
def test_products(gpu, rows, N, K, tile, gated):  # noqa: F811
    codes, scales, weights, weight_scales, bias = inputs_of(rows, N, K)
    n = N // 2 if gated else N
    y = torch.full((rows, n), 7.0, dtype=torch.bfloat16, device="cuda")
    gpu.spqt_i8_gemm(codes, scales, weights, weight_scales, y, bias=bias, gated=gated)
    if not gated:
        assert same(y, by_steps((codes, scales, weights, weight_scales, bias)).bfloat16())
        return
    for at in range(0, rows, 100000):
        part = torch.empty((min(100000, rows - at), n), dtype=torch.bfloat16, device="cuda")
        gpu.spqt_i8_gemm(codes[at : at + 100000], scales[at : at + 100000], weights, weight_scales, part, bias=bias, gated=True)
        assert same(y[at : at + 100000], part), at
