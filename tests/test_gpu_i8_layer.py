"""A prompt's layer in 8-bit integers whose products go by tiles and in parts: every call of it against its definition, in graphs, on streams and with one workspace for all."""
import pytest
import torch

from i8_paths import FEW, LAYER, PATHS, PROMPTS
from oracle import i8 as oracle
from test_gpu_i8 import PromptLayer, check_norm, gpu, rounded_to, same  # noqa: F401
from test_gpu_i8_ways import by_steps, inputs_of, sixteens

pytestmark = pytest.mark.gpu


class Recorded:
    """The package, with what norms and quantizations were given and gave."""

    def __init__(self, spqt):
        self.spqt, self.norms, self.quantized = spqt, [], []

    def __getattr__(self, name):
        return getattr(self.spqt, name)

    def spqt_i8_norm(self, h, gain, block=None, block_gain=None, residual=1.0, **outputs):
        given = {n: t.cpu() for n, t in (("h", h), ("gain", gain), ("block", block), ("block_gain", block_gain)) if t is not None}
        self.spqt.spqt_i8_norm(h, gain, block=block, block_gain=block_gain, residual=residual, **outputs)
        self.norms.append((given, {"residual": residual}, {n: t.clone() for n, t in outputs.items()}))

    def spqt_i8_quantize(self, x, codes, scales):
        self.spqt.spqt_i8_quantize(x, codes, scales)
        self.quantized.append((x.cpu(), codes.cpu(), scales.cpu()))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_every_call_of_a_layer(gpu, dtype):  # noqa: F811
    dtype = getattr(torch, dtype)
    recorded = Recorded(gpu)
    layer = PromptLayer(recorded, *LAYER, dtype)
    gen = torch.Generator().manual_seed(4)
    done = 0
    for rows in (PROMPTS[0], 1, PROMPTS[1]):
        recorded.norms, recorded.quantized = [], []
        h = torch.randn((rows, LAYER[0]), generator=gen).to(dtype).cuda()
        done += rows
        layer(h, torch.tensor([done], dtype=torch.int32, device="cuda"))
        assert len(recorded.norms) == 3 and len(recorded.quantized) == 2 and len(layer.seen) == 4
        for given, more, outputs in recorded.norms:
            check_norm(gpu, given, more, outputs, dtype)
        for x, codes, scales in recorded.quantized:
            want, want_scales = oracle.quantize(x)
            assert torch.equal(codes, want) and torch.equal(scales, want_scales)
        for name, codes, scales, y, gated in layer.seen:
            w, ws = layer.weights[name]
            if not gated:
                assert same(y, by_steps((codes, scales, w, ws, None)).to(dtype))
                continue
            assert same(y, sixteens(gpu, (codes, scales, w, ws, None), dtype))
            some = [0, rows // 2, rows - 1]
            want, off = oracle.product(codes[some].cpu(), scales[some].cpu(), w.cpu(), ws.cpu(), gated=True)
            assert rounded_to(y[some], want, off, dtype)


def test_a_layer_in_a_graph(gpu):  # noqa: F811
    """Replays with other inputs, with eager calls of another length in between, as the eager calls."""
    rows = PROMPTS[0]
    layer, other = PromptLayer(gpu, *LAYER, torch.bfloat16), PromptLayer(gpu, *LAYER, torch.bfloat16)
    gen = torch.Generator().manual_seed(5)
    inputs = [torch.randn((rows, LAYER[0]), generator=gen).bfloat16().cuda() for _ in range(3)]
    h, lengths = inputs[0].clone(), torch.tensor([rows], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(h, lengths)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            last = layer(h, lengths)
    torch.cuda.current_stream().wait_stream(side)
    for x in inputs + inputs[:2]:
        eager = x.clone()
        want = other(eager, lengths)
        h.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert same(last, want) and same(h, eager)
        layer.product("down", *products_inputs(gpu, layer, PROMPTS[1]))           # the graph's workspace, used by an eager call of another size
        torch.cuda.synchronize()


def products_inputs(gpu, layer, rows):  # noqa: F811
    codes, scales = gpu.new_i8_codes(rows, LAYER[4]), torch.rand(rows, device="cuda")
    codes.copy_(torch.randint(-127, 128, codes.shape, device="cuda", dtype=torch.int16).to(torch.int8))
    return codes, scales


@pytest.mark.parametrize("captured", [False, True])
def test_products_that_follow_each_other_on_one_workspace(gpu, captured):  # noqa: F811
    """Products in parts by all four tiles, gated and not, and others between them, one after the other on a stream of their own with one workspace, eager and in a graph; then with
    other inputs, the workspace full of anything."""
    sizes = [PATHS[tile, "parts"] for tile in ("64x128", "256x256", "128x128", "128x256")] + [FEW[2], PATHS["64x128", "rounds"]]
    sizes = sizes + sizes[::-1]
    largest = max(gpu.spqt_i8_workspace_bytes(*s) for s in sizes)
    space = torch.zeros(largest, dtype=torch.uint8, device="cuda")
    calls = []
    for i, (rows, N, K) in enumerate(sizes):
        gated = i % 3 == 1
        calls.append((inputs_of(rows, N, K, i), gated, torch.zeros((rows, N // 2 if gated else N), dtype=torch.float16 if i % 2 else torch.float32, device="cuda")))

    def run():
        for (codes, scales, weights, weight_scales, bias), gated, y in calls:
            gpu.spqt_i8_gemm(codes, scales, weights, weight_scales, y, bias=bias, gated=gated, workspace=space)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        side.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                run()
    for turn in range(3):
        for (codes, scales, weights, weight_scales, bias), _, y in calls:
            scales.mul_(1.0 + 0.25 * turn)
            codes[:, : codes.shape[1] // 2].neg_()
            y.fill_(7.0)
        space.fill_(85 * turn)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay() if captured else run()
        side.synchronize()
        for inputs, gated, y in calls:
            want = sixteens(gpu, inputs, y.dtype) if gated else by_steps(inputs).to(y.dtype)
            assert same(y, want), (turn, tuple(y.shape), gated)
