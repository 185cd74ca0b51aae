"""What the prompt side of a decoder is timed on, in 8-bit integers: where the sparse GEMVs take one token to four, a prompt or a
batch brings rows enough for a product of matrices.

A case is one call between two of a layer's products, or such a product:

    "quantize"  rows of 16-bit values to 8-bit codes with a scale for each row, and what the codes stand for
    "norm"      what a block has made joins the residual stream (normed, weighed channel by channel, with the stream's own scale, or
                plainly), the stream is normed for the next block, in 16 bits or in codes
    "gemm"      codes times weights in 8-bit integers with a scale for each token and each channel; "gated" ones have the gate's rows
                and the up projection's rows in one matrix and give silu(gate) * up

Sizes are those of decoders of 7B, 8B, 13B and 70B parameters, and generic ones.  Codes int8 [rows, K] and weights int8 [channels, K] have
rows that begin at multiples of 16 bytes; what lies behind the K-th byte of a row is anything.
"""
import math

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _gemm(name, rows, channels, K, dtype, gated=False, bias=False):
    case = {"kind": "gemm", "rows": rows, "channels": channels, "K": K, "dtype": dtype, "gated": gated, "bias": bias}
    return dict(case, name=name) if name else case


def _norm(name, rows, K, dtype, codes=True, block=True, block_gain=False, gate="none", residual=1.0, offset=0.0):
    case = {"kind": "norm", "rows": rows, "K": K, "dtype": dtype, "codes": codes, "block": block, "block_gain": block_gain, "gate": gate,
            "residual": residual, "offset": offset}
    return dict(case, name=name) if name else case


def _quantize(name, rows, K, dtype, wider=0):
    case = {"kind": "quantize", "rows": rows, "K": K, "dtype": dtype, "wider": wider}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token's q, k and v, 8B: all of it is reading the weights
        _gemm("gemm_token_8b", 1, 6144, 4096, "fp16"),
        # four drafted tokens through gate and up, 7B
        _gemm("gemm_drafts_7b", 4, 22016, 4096, "fp16", gated=True),
        # a server's batch through the down projection, 70B: many weights, few rows
        _gemm("gemm_batch_70b", 40, 8192, 28672, "bf16"),
        # a large batch, or a short prompt, 8B down
        _gemm("gemm_mid_8b", 250, 4096, 14336, "bf16"),
        # a prompt through gate and up, 8B
        _gemm("gemm_prompt_8b", 4001, 28672, 4096, "fp16", gated=True),
        # a chunk of a long prompt, 70B q, k and v
        _gemm("gemm_chunk_70b", 1024, 10240, 8192, "bf16"),
        # a head of odd sizes, its logits in 32 bits
        _gemm("gemm_odd_head", 777, 1111, 5003, "fp32", bias=True),
        # a decode step between two blocks, 8B: all latency
        _norm("norm_token_8b", 1, 4096, "fp16"),
        # a prompt, 70B width: the block's output is normed too and weighed channel by channel
        _norm("norm_prompt_70b", 4001, 8192, "bf16", block_gain=True, gate="channel"),
        # rows of an odd width, each with weights of its own, in 16 bits
        _norm("norm_odd", 333, 2111, "fp16", codes=False, gate="row", residual=0.75, offset=1.0),
        # a batch before the down projection, 70B
        _quantize("quantize_batch_70b", 40, 28672, "bf16"),
        # a prompt before the down projection, 8B
        _quantize("quantize_prompt_8b", 4001, 14336, "fp16"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


WIDTHS = [4096, 5120, 8192, 11008, 13824, 14336, 28672]


def draw(rng):
    """A case of the same ranges: any number of rows, widths of decoders and odd ones."""
    kind = rng.choice(["gemm", "gemm", "gemm", "norm", "quantize"])
    dtype = rng.choice(["fp16", "bf16"])
    if kind == "gemm":
        K = rng.choice(WIDTHS) if rng.random() < 0.5 else _spread(rng, 300, 29000)
        gated = rng.random() < 0.3
        channels = rng.choice(WIDTHS) if rng.random() < 0.5 else _spread(rng, 500, 29000)
        channels = max(500, min(channels, 230_000_000 // K))
        channels -= channels % 2 if gated else 0
        rows = min(_spread(rng, 1, 8000), int(4.6e11 / (K * channels)), 60_000_000 // channels)
        return _gemm(None, rows, channels, K, rng.choice(["fp16", "bf16", "bf16", "fp32"]), gated, rng.random() < 0.2)
    K = rng.choice(WIDTHS) if rng.random() < 0.5 else _spread(rng, 100, 28000)
    rows = min(_spread(rng, 1, 8000), (57_000_000 if kind == "quantize" else 24_000_000) // K)
    if kind == "quantize":
        return _quantize(None, rows, K, dtype, rng.choice([0, 0, 8, 104]))
    block = rng.random() < 0.8
    return _norm(None, rows, K, dtype, rng.random() < 0.6, block, block and rng.random() < 0.5, rng.choice(["none", "channel", "row"]) if block else "none",
                 rng.choice([1.0, 1.0, 0.5, 0.875]), rng.choice([0.0, 0.0, 1.0]))


# ------------------------------------------------------------------------------- inputs

def _codes(gen, rows, K):
    """int8 [rows, K] whose rows begin at multiples of 16 bytes, as large values of a row's normal ones leave them."""
    whole = torch.empty((rows, -(-K // 16) * 16), dtype=torch.int8, device="cuda")
    flat = whole.view(-1)
    for at in range(0, flat.numel(), 1 << 25):
        part = flat[at : at + (1 << 25)]
        part.copy_(torch.randn(part.shape, device="cuda", generator=gen, dtype=torch.float16).mul_(32).clamp_(-127, 127).round_())
    return whole[:, :K]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    rows, K, dtype = case["rows"], case["K"], TYPES[case["dtype"]]
    state = {"case": case}
    if case["kind"] == "gemm":
        channels = case["channels"]
        state["codes"], state["weights"] = _codes(gen, rows, K), _codes(gen, channels, K)
        state["scales"] = torch.exp(0.5 * normal(rows)) * 0.03
        state["weight_scales"] = torch.exp(0.2 * normal(channels)) * (0.03 / math.sqrt(K))
        state["bias"] = normal(channels) if case["bias"] else None
        state["y"] = torch.zeros((rows, channels // 2 if case["gated"] else channels), dtype=dtype, device="cuda")
        return state
    # some channels are larger than others
    loud = torch.exp(0.7 * normal(K))
    if case["kind"] == "norm":
        state["h"] = (normal(rows, K) * loud).to(dtype)
        state["gain"] = (1 - case["offset"] + 0.2 * normal(K)).to(dtype)
        state["block"] = (normal(rows, K) * torch.exp(0.4 * normal(K))).to(dtype) if case["block"] else None
        state["block_gain"] = (1 - case["offset"] + 0.2 * normal(K)).to(dtype) if case["block_gain"] else None
        state["gate"] = None if case["gate"] == "none" else (0.5 * (normal(K) if case["gate"] == "channel" else normal(rows, K))).to(dtype)
        state["h_out"] = torch.zeros_like(state["h"])
        state["out"] = torch.zeros_like(state["h"])
    else:
        # a slice of a wider tensor where the case says so
        state["x"] = (normal(rows, K + case["wider"]) * torch.cat([loud, loud.new_ones(case["wider"])])).to(dtype)[:, :K]
    state["codes"] = torch.zeros((rows, -(-K // 16) * 16), dtype=torch.int8, device="cuda")[:, :K]
    state["scales"] = torch.zeros(rows, device="cuda")
    state["values"] = torch.zeros((rows, K), dtype=dtype, device="cuda")
    return state


# ------------------------------------------------------------------------ the plain forms

EPS = 1e-5


def _held(x, dtype):
    """(what rows of numbers stand for once they are codes, the rows' scales)."""
    top = x.abs().amax(dim=1, keepdim=True).clamp(min=2.0 ** -100)
    scale, inverse, largest = top / 127.0, torch.full_like(top, 127.0) / top, torch.finfo(dtype).max
    values = torch.round(x * inverse) * scale
    return values.clamp(-largest, largest).to(dtype), scale[:, 0]


def _normed(x, gain, offset):
    return x * (1.0 / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS)) * (gain.float() + offset)


def _plain_norm(state):
    case = state["case"]
    dtype = TYPES[case["dtype"]]
    x = state["h"].float()
    result = {}
    if case["block"]:
        z = state["block"].float()
        if case["block_gain"]:
            z = _normed(z, state["block_gain"], case["offset"])
        if state["gate"] is not None:
            z = z * state["gate"].float()
        x = x * case["residual"] + z
        result["h"] = x.to(dtype)                # the next block's norm takes the sum before it is rounded
    x = _normed(x, state["gain"], case["offset"])
    if case["codes"]:
        result["values"], result["scales"] = _held(x, dtype)
    else:
        result["out"] = x.to(dtype)
    return result


def _plain_gemm(state):
    case = state["case"]
    y = torch.matmul(state["codes"].float(), state["weights"].float().t()) * state["scales"][:, None] * state["weight_scales"]
    if case["bias"]:
        y = y + state["bias"]
    if case["gated"]:
        g, u = y.chunk(2, dim=1)
        y = g / (1.0 + torch.exp(-g)) * u
    return {"y": y.to(TYPES[case["dtype"]])}


# --------------------------------------------------------------------------------- a pass

_space = None                                    # a program's one workspace, as large as its largest call asked for


def _workspace(spqt, case):
    global _space
    bytes_ = spqt.spqt_i8_workspace_bytes(case["rows"], case["channels"], case["K"])
    if _space is None or _space.numel() < bytes_:
        _space = spqt.new_i8_workspace(case["rows"], case["channels"], case["K"])
    return _space


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        if kind == "gemm":
            return _plain_gemm(state)
        if kind == "norm":
            return _plain_norm(state)
        return dict(zip(("values", "scales"), _held(state["x"].float(), TYPES[case["dtype"]])))
    import paper_2511_04477_amd as spqt
    if kind == "gemm":
        if "workspace" not in state:             # kept from call to call
            state["workspace"] = _workspace(spqt, case)
        spqt.spqt_i8_gemm(state["codes"], state["scales"], state["weights"], state["weight_scales"], state["y"], bias=state["bias"], gated=case["gated"],
                          workspace=state["workspace"])
        return {"y": state["y"]}
    result = {}
    if kind == "norm":
        given = {"codes": state["codes"], "scales": state["scales"]} if case["codes"] else {"out": state["out"]}
        if case["block"]:
            given.update(block=state["block"], block_gain=state["block_gain"], gate=state["gate"], residual=case["residual"], h_out=state["h_out"])
            result["h"] = state["h_out"]
        spqt.spqt_i8_norm(state["h"], state["gain"], eps=EPS, offset=case["offset"], **given)
        if not case["codes"]:
            return dict(result, out=state["out"])
    else:
        spqt.spqt_i8_quantize(state["x"], state["codes"], state["scales"])
    spqt.spqt_i8_read(state["codes"], state["scales"], state["values"])
    return dict(result, values=state["values"], scales=state["scales"])


# ----------------------------------------------------------------------------------- work

def work(case):
    rows, K = case["rows"], case["K"]
    if case["kind"] == "gemm":
        channels = case["channels"]
        made = rows * (channels // 2 if case["gated"] else channels) * (4 if case["dtype"] == "fp32" else 2)
        return {"bytes": (rows + channels) * (K + 4) + made + (4 * channels if case["bias"] else 0), "flops": 2 * rows * channels * K}
    back = 1 + 1 + 2                                                   # codes out, codes in, values out
    if case["kind"] == "quantize":
        return {"bytes": rows * (K * (2 + back) + 8), "flops": 4 * rows * K}
    each = 2 + (back if case["codes"] else 2) + (4 if case["block"] else 0) + (2 if case["gate"] == "row" else 0)
    shared = 1 + (1 if case["block_gain"] else 0) + (1 if case["gate"] == "channel" else 0)
    return {"bytes": rows * (K * each + (8 if case["codes"] else 0)) + 2 * K * shared, "flops": rows * K * (4 + (7 if case["block"] else 0))}


# ---------------------------------------------------------------------------- in 64 bits

def _exact_held(x):
    scale = x.abs().amax(dim=1, keepdim=True).clamp(min=2.0 ** -100) / 127
    return torch.round(x / scale) * scale, scale[:, 0]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "gemm":
        acc = torch.matmul(state["codes"].double(), state["weights"].double().t())
        y = acc * torch.outer(state["scales"].double(), state["weight_scales"].double())
        if case["bias"]:
            y += state["bias"].double()
        if case["gated"]:
            half = y.shape[1] // 2
            y = y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
        return {"y": y}
    if case["kind"] == "quantize":
        values, scales = _exact_held(state["x"].double())
        return {"values": values, "scales": scales}
    h = state["h"].double()
    result = {}

    def normed(x, gain):
        return x / torch.sqrt((x * x).sum(dim=1, keepdim=True) / case["K"] + EPS) * (gain.double() + case["offset"])

    if case["block"]:
        z = state["block"].double()
        if case["block_gain"]:
            z = normed(z, state["block_gain"])
        if state["gate"] is not None:
            z = z * state["gate"].double()
        h = result["h"] = case["residual"] * h + z
    x = normed(h, state["gain"])
    if not case["codes"]:
        return dict(result, out=x)
    result["values"], result["scales"] = _exact_held(x)
    return result
