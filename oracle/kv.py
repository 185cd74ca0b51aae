"""CPU oracle of the key/value cache in 8 bits.  TEST INFRASTRUCTURE ONLY.

Only the tests may import this module.  Plain loops over sequences, heads and blocks in 64-bit arithmetic (torch on the CPU,
for its bfloat16), from the definitions:

  scale(a)   the least number from a / 127 (2^-100 if that is more) on that has 12 significant bits, the last of them set; NaN if a
             is an infinity or a NaN
  code       x / scale rounded to the nearest integer
  a page     bytes code + 128: keys [token][element], values [element][place], place(t) = 16 (t / 4 % 4) + 4 (t / 16) + t % 4
  attention  s_t = scale q . k_t over the tokens that a row sees, p = exp(s - m) / sum, out = sum p_t v_t, lse = m + ln sum
  moving     (exactly) the scale of the largest |code * scale|, and code * (old scale / new scale), the quotient in fp32, to nearest, ties to even
  eviction   the last `recent` tokens and the heaviest others, the earlier one of two that weigh the same
"""
from __future__ import annotations

import math

import torch

BLOCK = 64
PLACE = [16 * (t // 4 % 4) + 4 * (t // 16) + t % 4 for t in range(BLOCK)]


def scale_of(largest: float) -> float:
    if not math.isfinite(largest):
        return math.nan
    mantissa, exponent = math.frexp(max(largest / 127.0, 2.0 ** -100))
    whole = math.ceil(mantissa * 4096)               # 2048 .. 4096
    if whole % 2 == 0:
        whole += 1
    if whole > 4096:
        whole = 4098                                 # 13 bits: the first one of the next power of two
    return math.ldexp(whole, exponent - 12)


def quantize(x):
    """x [tokens, dim] (64 bit) -> (codes int64, scale)."""
    if x.isnan().any() or x.isinf().any():
        return None, math.nan
    scale = scale_of(float(x.abs().max()))
    return torch.round(x / scale).long(), scale


def page_codes(page, which):
    """[64, dim] codes of one side of a page uint8 [2, 64, dim]."""
    side = page[which]
    if which == 0:
        return side.long() - 128
    return side.reshape(-1, BLOCK)[:, PLACE].t().long() - 128


def token_values(codes, scales, table_row, head, which, n):
    """fp64 [n, dim]: what the first n tokens of a sequence stand for."""
    found = []
    for b in range(-(-n // BLOCK)):
        page = int(table_row[b])
        found.append(page_codes(codes[page, head], which).double() * float(scales[page, head, which]))
    dim = codes.shape[-1]
    return torch.cat(found)[:n] if found else torch.zeros((0, dim), dtype=torch.float64)


def rounded(x, dtype):
    largest = torch.finfo(dtype).max
    return x.clamp(-largest, largest).to(dtype)


def attention(codes, scales, table, lengths, q, counts, scale, window):
    """out, lse and, for every sequence and kv head, the sums of probabilities [tokens], all in 64 bits; and two bounds:
    `sway` how far a score may be off in units of fp32 rounding (sum of |q| |k| times scale), `spread` sum p |v|."""
    S, n, Hq, dim = q.shape
    H = codes.shape[1]
    out = torch.zeros((S, n, Hq, dim), dtype=torch.float64)
    lse = torch.full((S, n, Hq), -math.inf, dtype=torch.float64)
    sway = torch.zeros((S, n, Hq), dtype=torch.float64)
    spread = torch.zeros((S, n, Hq, dim), dtype=torch.float64)
    weights, weight_sway = [], []
    for s in range(S):
        L, c = int(lengths[s]), int(counts[s])
        per_head, per_sway = [], []
        for h in range(H):
            k, v = (token_values(codes, scales, table[s], h, which, L) for which in (0, 1))
            sums, sways = torch.zeros(L, dtype=torch.float64), torch.zeros(L, dtype=torch.float64)
            for i in range(c):
                at = L - c + i
                low = max(0, at - window + 1) if window > 0 else 0
                if at < 0 or at < low:
                    continue
                for j in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    x = (k[low : at + 1] @ q[s, i, j].double()) * scale
                    lse[s, i, j] = torch.logsumexp(x, 0)
                    p = torch.exp(x - lse[s, i, j])
                    out[s, i, j] = p @ v[low : at + 1]
                    spread[s, i, j] = p @ v[low : at + 1].abs()
                    sway[s, i, j] = float((k[low : at + 1].abs() @ q[s, i, j].double().abs()).max()) * scale
                    sums[low : at + 1] += p
                    sways[low : at + 1] += p * sway[s, i, j]
            per_head.append(sums)
            per_sway.append(sways)
        weights.append(per_head)
        weight_sway.append(per_sway)
    return out, lse, weights, sway, spread, weight_sway


def requantize(parts):
    """(codes [tokens, dim], their scale) of one head, several blocks' tokens -> (codes, scale) as one block, from code * scale as it is; None and NaN where a scale is none."""
    if any(math.isnan(s) for _, s in parts):
        return None, math.nan
    scale = scale_of(max(float(c.abs().max()) * s for c, s in parts))
    ratio = lambda s: (torch.tensor(s, dtype=torch.float32) / torch.tensor(scale, dtype=torch.float32)).clamp(max=128.0).double()  # noqa: E731
    return torch.cat([torch.round(c.double() * ratio(s)) for c, s in parts]).long(), scale


def choose(weights, length, keep, recent):
    """Kept positions, ascending; weights [length]."""
    late = min(recent, length)
    order = sorted(range(length - late), key=lambda t: (not math.isnan(float(weights[t])), -float(weights[t]) if not math.isnan(float(weights[t])) else 0.0, t))
    return sorted(order[: min(length, keep) - late]) + list(range(length - late, length))
