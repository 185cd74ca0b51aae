"""What the cache operators are timed on: a decoder's keys and values held in 8 bits, from the append of new tokens over the
attention that reads them to the eviction of what attention no longer weighs.

A case is one call of a decoder layer: "append" (quantize new tokens into the cache, and read them back as 16-bit values),
"attend" (attention of 1 to some thousand query rows per sequence over the cache, with or without the accumulated weights) or
"evict" (keep the heaviest and the latest tokens, move them to other pages).  Head counts are those of decoders of 7B, 8B, 13B
and 70B parameters with heads of 128, and generic ones (one head shared by all, heads of 64 and 256).

The cache is paged: `codes` uint8 [pages, kv heads, 2, 64, dim] holds 64 tokens of a page, code + 128, keys as [token][dim] and
values as [dim][place of token], place 16 * (t / 4 % 4) + 4 * (t / 16) + t % 4; `scales` fp32 [pages, kv heads, 2];
`tail` the 16-bit values of every sequence's last block; `table` int32 [sequences, blocks] and `lengths` int32 [sequences], which
count the tokens that the cache holds once the call is done.
"""
import math

import torch

own = False

BLOCK = 64
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _append(name, q_heads, kv_heads, dim, dtype, seqs, low, high, rows, idle=0):
    case = {"kind": "append", "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "seqs": seqs, "low": low, "high": high,
            "rows": rows, "idle": idle}
    return dict(case, name=name) if name else case


def _attend(name, q_heads, kv_heads, dim, dtype, seqs, low, high, rows, idle=0, window=0, weigh=False, decay=1.0):
    case = {"kind": "attend", "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "seqs": seqs, "low": low, "high": high,
            "rows": rows, "idle": idle, "window": window, "weigh": weigh, "decay": decay}
    return dict(case, name=name) if name else case


def _evict(name, kv_heads, dim, dtype, seqs, low, high, keep, recent):
    case = {"kind": "evict", "q_heads": kv_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "seqs": seqs, "low": low, "high": high,
            "rows": 1, "idle": 0, "keep": keep, "recent": recent}
    return dict(case, name=name) if name else case


def listed():
    return [
        # a decode step's new token for four sequences of an 8B decoder: all latency
        _append("append_token", 32, 8, 128, "fp16", 4, 200, 9000, 1),
        # prompts of uneven lengths behind what the sequences hold already, 70B heads
        _append("append_prompts", 64, 8, 128, "bf16", 6, 1100, 9001, 6007),
        # a chat's first tokens, one sequence, 8B: the smallest attention
        _attend("step_short_8b", 32, 8, 128, "fp16", 1, 333, 333, 1),
        # 7B: every query head has keys of its own
        _attend("step_7b", 32, 32, 128, "fp16", 1, 4095, 4095, 1),
        # one long document, 70B
        _attend("step_long_70b", 64, 8, 128, "bf16", 1, 131000, 131000, 1),
        # a server's batch: uneven lengths, five slots idle
        _attend("step_batch_8b", 32, 8, 128, "bf16", 40, 17, 9500, 1, idle=5),
        # 13B, four drafted tokens per sequence, each seeing the last 2000
        _attend("step_drafts_13b", 40, 40, 128, "fp16", 3, 1500, 7777, 4, window=2000),
        # a decode step that also accumulates what every cached token weighed
        _attend("step_weighed_8b", 32, 8, 128, "fp16", 2, 9000, 16001, 1, weigh=True),
        # a whole prompt, 8B
        _attend("prompt_8b", 32, 8, 128, "fp16", 1, 4001, 4001, 4001),
        # a chunk of a long prompt, 70B
        _attend("chunk_70b", 64, 8, 128, "bf16", 1, 32768, 32768, 1024),
        # two caches of a long prompt cut down to a budget
        _evict("evict_prompts", 8, 128, "bf16", 2, 20000, 33001, 8192, 512),
        # a step over the budget of one sequence: many heads, little to drop
        _evict("evict_step_7b", 32, 128, "fp16", 1, 2300, 2300, 2048, 256),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


HEADS = [(32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (32, 8, 128), (64, 8, 128), (16, 1, 128), (12, 4, 64), (16, 2, 256), (25, 5, 64), (8, 8, 192)]


def draw(rng):
    """A case of the same ranges: any head counts, type, lengths from one token on, idle slots."""
    q_heads, kv_heads, dim = rng.choice(HEADS)
    dtype = rng.choice(["fp16", "bf16"])
    kind = rng.choice(["append", "attend", "attend", "attend", "attend", "evict"])
    per_token = 2 * kv_heads * dim                     # bytes of codes
    if kind == "append":
        rows = _spread(rng, 1, 6000)
        seqs = max(1, min(_spread(rng, 1, 48), 70_000_000 // (per_token * rows)))
        high = rows + _spread(rng, 1, 8000)
        return _append(None, q_heads, kv_heads, dim, dtype, seqs, rng.randint(rows, high), high, rows, rng.choice([0, 0, 1]) if seqs > 1 else 0)
    if kind == "evict":
        high = _spread(rng, 700, 33000)
        seqs = max(1, min(_spread(rng, 1, 16), 140_000_000 // (per_token * high)))
        keep = max(64, int(high * rng.uniform(0.1, 0.95)))
        return _evict(None, kv_heads, dim, dtype, seqs, rng.randint(high // 3, high), high, keep, rng.randint(0, keep // 2))
    form = rng.choice(["step", "step", "drafts", "chunk"])
    if form == "chunk":
        rows = _spread(rng, 40, 4000)
        high = rows + _spread(rng, 1, 30000)
        pairs = q_heads * dim * rows * high
        seqs = max(1, min(_spread(rng, 1, 6), int(2.2e11 / pairs)))
        while pairs > 2.2e11:
            rows, high = max(1, rows // 2), max(rows, high * 2 // 3)
            pairs = q_heads * dim * rows * high
    else:
        rows = 1 if form == "step" else rng.randint(2, 12)
        high = _spread(rng, 2 * rows, 130000)
        seqs = max(1, min(_spread(rng, 1, 64), 260_000_000 // (per_token * high)))
    low = rng.randint(rows, high) if seqs > 1 else high
    weigh = rng.random() < 0.3
    window = _spread(rng, 16, high) if high > 16 and rng.random() < 0.25 else 0
    return _attend(None, q_heads, kv_heads, dim, dtype, seqs, low, high, rows, rng.choice([0, 0, 1]) if seqs > 1 else 0, window, weigh,
                   rng.choice([1.0, 1.0, 0.0, 0.9]) if weigh else 1.0)


def _lengths(case):
    """Tokens and new rows of every sequence: the first one is the longest, the last `idle` ones are empty."""
    n, low, high, rows = case["seqs"], case["low"], case["high"], case["rows"]
    lengths, counts = [], []
    for s in range(n):
        part = 1.0 if s == 0 else (s * 0.6180339887) % 1.0
        lengths.append(low + int((high - low) * part))
        counts.append(min(lengths[-1], max(1, int(rows * (1.0 if s == 0 else 0.5 + 0.5 * part)))))
        if s >= n - case["idle"]:
            lengths[-1] = counts[-1] = 0
    return lengths, counts


# ------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    lengths, counts = _lengths(case)
    seqs, rows, dim, kv_heads, q_heads = case["seqs"], case["rows"], case["dim"], case["kv_heads"], case["q_heads"]
    dtype = TYPES[case["dtype"]]
    blocks = max(1, -(-max(lengths) // BLOCK))
    new_blocks = -(-case["keep"] // BLOCK) if case["kind"] == "evict" else 0
    pages = seqs * blocks + 3
    state = {"case": case, "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
             "counts": torch.tensor(counts, dtype=torch.int32, device="cuda") if seqs > 1 else None, "scale": 1.0 / math.sqrt(dim)}
    # the pages of a sequence lie anywhere in the pool
    order = torch.randperm(pages, device="cuda", generator=gen)[: seqs * blocks]
    state["table"] = order.view(seqs, blocks).to(torch.int32).contiguous()
    total = pages + seqs * new_blocks
    codes = torch.full((total, kv_heads, 2, BLOCK, dim), 128, dtype=torch.uint8, device="cuda")
    for p in range(0, pages, 512):
        part = codes[p : p + 512]
        part.copy_(torch.randn(part.shape, device="cuda", generator=gen, dtype=torch.float16).mul_(38).clamp_(-127, 127).round_().add_(128))
    state["codes"] = codes
    state["scales"] = torch.rand((total, kv_heads, 2), device="cuda", generator=gen) * 0.02 + 0.01
    if case["kind"] != "attend":
        state["tail"] = torch.zeros((seqs, kv_heads, 2, BLOCK, dim), dtype=dtype, device="cuda")
    if case["kind"] == "evict":
        # sums of probabilities over many steps: most tokens hardly any, a few much
        state["weights"] = torch.zeros((total, kv_heads, BLOCK), device="cuda")
        state["weights"][:pages] = torch.exp(2.5 * normal(pages, kv_heads, BLOCK)) * 1e-2
        state["new_table"] = torch.arange(pages, total, dtype=torch.int32, device="cuda").view(seqs, new_blocks)
        state["new_lengths"] = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        state["kept"] = torch.zeros((seqs, kv_heads, case["keep"]), dtype=torch.int32, device="cuda")
        for name in ("k_out", "v_out"):
            state[name] = torch.zeros((seqs, case["keep"], kv_heads, dim), dtype=dtype, device="cuda")
        return state
    # q, k and v as one projection gives them, side by side
    qkv = normal(seqs, rows, q_heads + 2 * kv_heads, dim)
    qkv *= torch.exp(0.5 * normal(1, 1, q_heads + 2 * kv_heads, dim))        # some channels are larger than others
    qkv = qkv.to(dtype)
    state["q"], state["k"], state["v"] = qkv.split([q_heads, kv_heads, kv_heads], dim=2)
    if case["kind"] == "attend":
        state["out"] = torch.zeros((seqs, rows, q_heads, dim), dtype=dtype, device="cuda")
        state["lse"] = torch.zeros((seqs, rows, q_heads), device="cuda")
        if case["weigh"]:
            state["weights"] = torch.exp(2.5 * normal(total, kv_heads, BLOCK)) * 1e-2
            state["weights_before"] = state["weights"].clone()
        return state
    # an open block has the values that its codes came from, and the scale that they ask for
    old = (state["lengths"] - torch.tensor(counts, dtype=torch.int32, device="cuda")).long()
    state["tail"].copy_(normal(seqs, kv_heads, 2, BLOCK, dim) * 0.7)
    inside = (torch.arange(BLOCK, device="cuda") < (old % BLOCK)[:, None])[:, None, None, :, None]
    state["tail"] *= inside
    at = torch.gather(state["table"].long(), 1, (old // BLOCK).clamp(max=blocks - 1)[:, None])[:, 0]
    scale = _scale_of(state["tail"].float().abs().amax(dim=(3, 4)))
    open_codes = torch.round(state["tail"].float() / scale[..., None, None]).add_(128).to(torch.uint8)
    some = (old % BLOCK) > 0
    codes[at[some], :, 0] = open_codes[some][:, :, 0]
    codes[at[some], :, 1] = _placed(open_codes[some][:, :, 1])
    state["scales"][at[some]] = scale[some]
    state["weights"] = normal(total, kv_heads, BLOCK)
    # what is read back: the blocks that the call writes to, whole
    state["read_counts"] = (state["lengths"] - old // BLOCK * BLOCK).to(torch.int32) * (state["lengths"] > 0)
    for name in ("k_out", "v_out"):
        state[name] = torch.zeros((seqs, rows + BLOCK - 1, kv_heads, dim), dtype=dtype, device="cuda")
    return state


# ------------------------------------------------------------------------ the plain forms

def _scale_of(largest):
    """The scale of a block: the least number from largest / 127 on that has 12 significant bits, the last of them set."""
    bits = torch.clamp(largest / 127.0, min=2.0 ** -100).contiguous().view(torch.int32)
    odd = (bits & ~0x1FFF) | 0x1000
    return torch.where(odd < bits, odd + 0x2000, odd).view(torch.float32)


def _placed(values):
    """[..., 64 tokens, dim] in the order in which a page holds values: [..., dim, place] with the shape of the argument."""
    lead, dim = values.shape[:-2], values.shape[-1]
    t = values.reshape(*lead, 4, 4, 4, dim)               # 16s of tokens, 4s in them, token
    n = len(lead)
    return t.permute(*range(n), n + 3, n + 1, n, n + 2).reshape(*lead, BLOCK, dim)


def _cached(state, which):
    """fp32 [sequences, kv heads, blocks * 64, dim] of the keys (0) or values (1)."""
    dim = state["case"]["dim"]
    table = state["table"].long()
    c = state["codes"][table, :, which].float() - 128.0                  # [S, B, H, 64, dim]
    if which:
        S, B, H = c.shape[:3]
        c = c.reshape(S, B, H, dim, 4, 4, 4).permute(0, 1, 2, 5, 4, 6, 3).reshape(S, B, H, BLOCK, dim)
    c = c * state["scales"][table][..., which, None, None]
    return c.transpose(1, 2).flatten(2, 3)


def _counts(state):
    return state["counts"] if state["counts"] is not None else torch.clamp(state["lengths"], max=state["case"]["rows"])


def _plain_attend(state):
    case = state["case"]
    S, n, H, dim = case["seqs"], case["rows"], case["kv_heads"], case["dim"]
    group = case["q_heads"] // H
    k, v = _cached(state, 0), _cached(state, 1)
    q = state["q"].float().view(S, n, H, group, dim).permute(0, 2, 1, 3, 4).reshape(S, H, n * group, dim)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * state["scale"]
    lengths, counts = state["lengths"].long(), _counts(state).long()
    row = torch.arange(n, device="cuda").repeat_interleave(group)
    at = (lengths - counts)[:, None] + row                                # position of every row
    t = torch.arange(k.shape[2], device="cuda")
    seen = (t <= at[..., None]) & (row < counts[:, None])[..., None]
    if case["window"]:
        seen &= t > (at - case["window"])[..., None]
    s = s.masked_fill_(~seen[:, None], -math.inf)
    top = s.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    some = torch.where(total > 0, total, torch.ones_like(total))
    p = p.div_(some)
    out = torch.matmul(p, v)
    lse = torch.where(total > 0, top + some.log(), torch.full_like(top, -math.inf))
    back = lambda x: x.reshape(S, H, n, group, -1).permute(0, 2, 1, 3, 4).reshape(S, n, H * group, -1)  # noqa: E731
    result = {"out": back(out).to(TYPES[case["dtype"]]), "lse": back(lse)[..., 0]}
    if case["weigh"]:
        sums = p.sum(dim=2).view(S, H, -1, BLOCK).transpose(1, 2)         # [S, blocks, H, 64]
        w = state["weights_before"].clone()
        table = state["table"].long()
        inside = (t.view(1, -1, 1, BLOCK) < lengths.view(S, 1, 1, 1))
        before = w[table]
        w[table] = torch.where(inside, case["decay"] * before + sums, before)
        result["weights"] = w
    return result


def _rounded(values, dtype):
    """Cached values as a reader gets them."""
    largest = torch.finfo(dtype).max
    return values.clamp(-largest, largest).to(dtype)


def _quantized(blocks, dtype):
    """(what [..., 64, dim] blocks stand for once they are held in 8 bits, their scales)."""
    scale = _scale_of(blocks.abs().amax(dim=(-2, -1)))
    held = torch.round(blocks / scale[..., None, None]) * scale[..., None, None]
    return _rounded(held, dtype), scale


def _plain_append(state):
    case = state["case"]
    S, n, H, dim = case["seqs"], case["rows"], case["kv_heads"], case["dim"]
    dtype = TYPES[case["dtype"]]
    lengths, counts = state["lengths"].long(), _counts(state).long()
    old = lengths - counts
    first = old // BLOCK
    blocks = (n + BLOCK - 2) // BLOCK + 1
    slot = torch.arange(blocks * BLOCK, device="cuda")
    at = first[:, None] * BLOCK + slot                                    # position of every slot
    given = (at - old[:, None]).clamp(0, n - 1)[..., None, None].expand(-1, -1, H, dim)
    held = state["tail"].float()[:, :, :, slot % BLOCK]                   # [S, H, 2, slots, dim]
    result, scales = {}, state["scales"].clone()
    table = state["table"].long()
    block = first[:, None] + torch.arange(blocks, device="cuda")
    page = torch.gather(table, 1, block.clamp(max=table.shape[1] - 1))
    live = (block * BLOCK < lengths[:, None]) & (counts > 0)[:, None]
    for which, name in ((0, "k"), (1, "v")):
        x = torch.gather(state[name].float(), 1, given).transpose(1, 2)   # [S, H, slots, dim]
        x = torch.where((at < old[:, None])[:, None, :, None], held[:, :, which], x)
        x = x * ((at < lengths[:, None]) & (counts > 0)[:, None])[:, None, :, None]
        values, scale = _quantized(x.view(S, H, blocks, BLOCK, dim), dtype)
        result[name] = values.flatten(2, 3).transpose(1, 2)[:, : n + BLOCK - 1].contiguous()
        scales[page[live], :, which] = scale.transpose(1, 2)[live]
    result["scales"] = scales
    return result


def _plain_evict(state):
    case = state["case"]
    S, H, dim, keep, recent = case["seqs"], case["kv_heads"], case["dim"], case["keep"], case["recent"]
    dtype = TYPES[case["dtype"]]
    lengths = state["lengths"].long()
    table = state["table"].long()
    w = state["weights"][table].transpose(1, 2).flatten(2, 3)             # [S, H, tokens]
    t = torch.arange(w.shape[2], device="cuda")
    key = torch.where(t >= (lengths - recent)[:, None], math.inf, 0.0)[:, None] + w
    key = torch.where((t < lengths[:, None])[:, None], key, -math.inf)
    ranked = torch.sort(key, dim=2, descending=True, stable=True).indices
    new = lengths.clamp(max=keep)
    slots = min(keep, w.shape[2])
    there = (torch.arange(slots, device="cuda") < new[:, None])[:, None]
    index = torch.where(there, ranked[:, :, :slots], 1 << 30).sort(dim=2).values
    kept = torch.full((S, H, keep), -1, dtype=torch.int32, device="cuda")
    kept[:, :, :slots] = torch.where(there, index, -1)
    at = torch.where(there, index, 0)
    blocks = -(-keep // BLOCK)
    result = {"kept": kept, "lengths": new.to(torch.int32)}
    moved = torch.zeros((S, H, blocks * BLOCK), device="cuda")
    moved[:, :, :slots] = torch.gather(w, 2, at) * there
    result["weights"] = moved.view(S, H, blocks, BLOCK).transpose(1, 2).flatten(0, 1).contiguous()
    for which, name in ((0, "k"), (1, "v")):
        x = _rounded(torch.gather(_cached(state, which), 2, at[..., None].expand(-1, -1, -1, dim)), dtype).float()
        full = torch.zeros((S, H, blocks * BLOCK, dim), device="cuda")
        full[:, :, :slots] = x * there[..., None]
        values, _ = _quantized(full.view(S, H, blocks, BLOCK, dim), dtype)
        values = values.flatten(2, 3)[:, :, :keep]                         # as read back: the last token in the last of its rows
        result[name] = values.transpose(1, 2).contiguous()
    return result


# --------------------------------------------------------------------------------- a pass

_space = None                                    # a program's one workspace, as large as its largest call asked for


def _workspace(spqt, case, blocks):
    global _space
    bytes_ = spqt.spqt_kv_workspace_bytes(case["seqs"], case["rows"], case["q_heads"], case["kv_heads"], case["dim"], blocks)
    if _space is None or _space.numel() < bytes_:
        _space = spqt.new_kv_workspace(case["seqs"], case["rows"], case["q_heads"], case["kv_heads"], case["dim"], blocks)
    return _space


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[kind](state)
    import paper_2511_04477_amd as spqt
    codes, scales, table, lengths = state["codes"], state["scales"], state["table"], state["lengths"]
    if kind == "attend":
        if "workspace" not in state:             # kept from call to call
            state["workspace"] = _workspace(spqt, case, table.shape[1])
        weights = None
        if case["weigh"]:
            weights = state["weights"]
            weights.copy_(state["weights_before"])          # every pass starts from the same sums
        spqt.spqt_kv_attention(codes, scales, table, lengths, state["q"], state["out"], state["workspace"], scale=state["scale"],
                               counts=state["counts"], window=case["window"], lse=state["lse"], weights=weights, decay=case["decay"])
        result = {"out": state["out"], "lse": state["lse"]}
        return result if weights is None else dict(result, weights=weights)
    if kind == "append":
        spqt.spqt_kv_append(codes, scales, state["tail"], table, lengths, state["k"], state["v"], counts=state["counts"], weights=state["weights"])
        spqt.spqt_kv_read(codes, scales, table, lengths, state["k_out"], state["v_out"], counts=state["read_counts"])
        return {"k": state["k_out"], "v": state["v_out"], "scales": scales}
    spqt.spqt_kv_evict(codes, scales, state["tail"], state["weights"], table, lengths, case["keep"], case["recent"], state["new_table"],
                       state["new_lengths"], state["kept"])
    spqt.spqt_kv_read(codes, scales, state["new_table"], state["new_lengths"], state["k_out"], state["v_out"], counts=state["new_lengths"])
    moved = state["weights"][state["weights"].shape[0] - state["new_table"].numel() :]
    return {"kept": state["kept"], "lengths": state["new_lengths"], "weights": moved, "k": state["k_out"], "v": state["v_out"]}


# ----------------------------------------------------------------------------------- work

def work(case):
    lengths, counts = _lengths(case)
    H, Hq, dim = case["kv_heads"], case["q_heads"], case["dim"]
    tokens, new = sum(lengths), sum(counts)
    if case["kind"] == "append":
        # 16-bit keys and values in, codes out; codes in, 16-bit values out
        return {"bytes": new * H * dim * 2 * (2 + 1 + 1 + 2) + new * H * 4, "flops": 2 * new * H * dim * 2}
    if case["kind"] == "evict":
        moved = sum(min(n, case["keep"]) for n in lengths)
        return {"bytes": H * (4 * tokens + moved * (2 * dim * (1 + 1 + 1 + 2) + 4 + 8)), "flops": H * tokens + 4 * moved * H * dim}
    window = case["window"] or 1 << 40
    pairs = read = 0
    for n, c in zip(lengths, counts):
        read += n - max(0, n - c + 1 - window) if c else 0
        full = max(0, n - c + 1 - window) if c else 0            # where the first row's view begins
        pairs += c * (n - c) + c * (c + 1) // 2 if full == 0 and n <= window else sum(min(window, n - c + i + 1) for i in range(c))
    total = read * H * (2 * dim + 8 / BLOCK) + new * Hq * (4 * dim + 4)
    if case["weigh"]:
        total += tokens * H * (8 if case["decay"] else 4)
    return {"bytes": total, "flops": 4 * dim * Hq * pairs}


# ---------------------------------------------------------------------- the same in 64 bits

def _exact_scale(largest):
    mantissa, exponent = torch.frexp(torch.clamp(largest / 127.0, min=2.0 ** -100))
    whole = torch.ceil((mantissa * 4096 - 1) / 2) * 2 + 1                # the next odd number of 12 bits
    whole = torch.where(whole > 4096, torch.full_like(whole, 4098.0), whole)
    return torch.ldexp(whole, exponent - 12)


def _exact_tokens(state, s, h, which, index):
    """fp64 [len(index), dim]: tokens of one sequence and head, from their codes."""
    page = state["table"][s].long()[index // BLOCK]
    t = index % BLOCK
    if which == 0:
        code = state["codes"][page, h, 0, t].double()
    else:
        place = 16 * (t // 4 % 4) + 4 * (t // 16) + t % 4
        flat = state["codes"][:, h, 1].reshape(state["codes"].shape[0], -1, BLOCK)
        code = flat[page, :, place].double()
    return (code - 128) * state["scales"][page, h, which].double()[:, None]


def _exact_held(values):
    """fp64 [tokens, dim] of one head, 64 tokens a block, as the cache then holds them; and the blocks' scales."""
    out, scales = [], []
    for part in values.split(BLOCK):
        scale = _exact_scale(part.abs().max())
        out.append(torch.round(part / scale) * scale)
        scales.append(scale)
    return torch.cat(out), torch.stack(scales)


def exact(case, seed):
    lengths, counts = _lengths(case)
    H, dim = case["kv_heads"], case["dim"]
    if sum(lengths) * H > 3_000_000 or (case["kind"] != "attend" and sum(lengths) * H > 700_000):
        return None
    state = prepare(case, seed)
    dtype, device = TYPES[case["dtype"]], "cuda"
    largest = torch.finfo(dtype).max
    if case["kind"] == "append":
        result = {name: torch.zeros(state["k_out"].shape, dtype=torch.float64, device=device) for name in ("k", "v")}
        scales = state["scales"].double()
        for s, (n, c) in enumerate(zip(lengths, counts)):
            if not c:
                continue
            before = (n - c) % BLOCK
            page = state["table"][s].long()[(n - c) // BLOCK : (n - 1) // BLOCK + 1]
            for h in range(H):
                for which, name in ((0, "k"), (1, "v")):
                    x = torch.cat([state["tail"][s, h, which, :before], state[name][s, :c, h]]).double()
                    held, scale = _exact_held(x)
                    result[name][s, : c + before, h] = held.clamp(-largest, largest)
                    scales[page, h, which] = scale
        return dict(result, scales=scales)
    if case["kind"] == "evict":
        keep, recent = case["keep"], case["recent"]
        result = {name: torch.zeros(state["k_out"].shape, dtype=torch.float64, device=device) for name in ("k", "v")}
        weights = torch.zeros((case["seqs"], -(-keep // BLOCK) * BLOCK, H), dtype=torch.float64, device=device)
        for s, n in enumerate(lengths):
            for h in range(H):
                w = state["weights"][state["table"][s].long(), h].reshape(-1)[:n].double()
                older = max(0, n - recent)
                chosen = torch.sort(w[:older], descending=True, stable=True).indices[: min(n, keep) - (n - older)]
                index = torch.cat([chosen.sort().values, torch.arange(older, n, device=device)])
                weights[s, : len(index), h] = w[index]
                for which, name in ((0, "k"), (1, "v")):
                    x = _exact_tokens(state, s, h, which, index).clamp(-largest, largest).to(dtype).double()
                    result[name][s, : len(index), h] = _exact_held(x)[0].clamp(-largest, largest)
        weights = weights.view(case["seqs"], -1, BLOCK, H).transpose(2, 3).flatten(0, 1)
        return dict(result, kept=None, lengths=None, weights=weights)
    Hq, rows, window = case["q_heads"], case["rows"], case["window"] or 1 << 40
    out = torch.zeros((case["seqs"], rows, Hq, dim), dtype=torch.float64, device=device)
    lse = torch.full((case["seqs"], rows, Hq), -math.inf, dtype=torch.float64, device=device)
    weights = state["weights_before"].double() if case["weigh"] else None
    for s, (n, c) in enumerate(zip(lengths, counts)):
        if not n:
            continue
        t = torch.arange(n, device=device)
        blocks = -(-n // BLOCK)
        page = state["table"][s].long()[:blocks]
        for h in range(H):
            sums = torch.zeros(blocks * BLOCK, dtype=torch.float64, device=device)
            k, v = (_exact_tokens(state, s, h, which, t) for which in (0, 1))
            for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                x = torch.mm(state["q"][s, :c, g].double(), k.t().contiguous()) * (1.0 / math.sqrt(dim))
                at = n - c + torch.arange(c, device=device)[:, None]
                x[(t > at) | (t <= at - window)] = -math.inf
                lse[s, :c, g] = torch.logsumexp(x, dim=1)
                p = torch.exp(x - lse[s, :c, g, None])
                out[s, :c, g] = torch.mm(p, v)
                sums[:n] += p.sum(dim=0)
            if weights is not None:
                w = weights[page, h].reshape(-1)
                weights[page, h] = torch.where(torch.arange(blocks * BLOCK, device=device) < n, case["decay"] * w + sums, w).view(blocks, BLOCK)
    result = {"out": out, "lse": lse}
    return result if weights is None else dict(result, weights=weights)
