"""A decoder layer's attention half on this library: sparse int4 projections, the key/value cache in 8 bits, and its eviction.

    python examples/decode_layer.py [--hidden 4096 --q-heads 32 --kv-heads 8 --prompt 500 --steps 300 --budget 512 --recent 64]

Random weights and hidden states stand in for a model's.  The prompt goes through the layer four tokens at a time, the steps one by one: q, k and v of the
columns that the threshold keeps (spqt_gemv_fused_rows, spqt_gemv_fused), rotated positions, append, attention with the accumulated weights, output projection.
When the cache is 64 tokens over its budget, what attention weighed least is dropped and the rest moves to other pages.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_04477_amd as spqt  # noqa: E402


class Layer:
    def __init__(self, hidden, q_heads, kv_heads, head_dim, budget, recent, sparsity, seed=0):
        r = np.random.default_rng(seed)
        self.hidden, self.q_heads, self.kv_heads, self.head_dim = hidden, q_heads, kv_heads, head_dim
        self.budget, self.recent = budget, recent
        width = (q_heads + 2 * kv_heads) * head_dim
        self.shapes = {"qkv": (width, hidden), "o": (hidden, q_heads * head_dim)}
        self.weights, self.spaces = {}, {}
        for name, (M, K) in self.shapes.items():
            q = r.integers(0, 256, (M, K // 2), dtype=np.uint8)
            scales = r.uniform(0.5, 1.5, (M, K // 128)) * (0.3 / np.sqrt(K))
            self.weights[name] = torch.from_numpy(spqt.spqt_pack(q, scales.astype(np.float16))).cuda()
            self.spaces[name] = spqt.new_workspace(M, K, 4)
        # |x| of the hidden states and of attention's outputs are not known here: a quantile of a normal distribution's for the former, none dropped for the latter
        self.threshold = float(np.quantile(np.abs(r.standard_normal(1 << 16)), sparsity))
        # pages for the sequence and, while it is cut down, for its successor
        self.blocks = -(-(budget + 64 + 4) // 64)
        pages = 2 * self.blocks
        self.codes, self.scales, self.tail, self.seen = spqt.new_kv_cache(pages, kv_heads, head_dim, 1, torch.float16, weights=True)
        tables = torch.arange(pages, dtype=torch.int32, device="cuda").view(2, 1, self.blocks)
        self.table, self.spare = tables[0].contiguous(), tables[1].contiguous()
        self.lengths, self.new_lengths = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        self.kept = torch.zeros((1, kv_heads, budget), dtype=torch.int32, device="cuda")
        self.space = spqt.new_kv_workspace(1, 4, q_heads, kv_heads, head_dim, self.blocks)
        self.in_cache, self.position, self.evictions = 0, 0, 0
        self.frequencies = 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda") / head_dim)

    def project(self, name, x, threshold):
        M, K = self.shapes[name]
        y = torch.empty((x.shape[0], M), dtype=torch.float16, device="cuda")
        if x.shape[0] == 1:
            spqt.spqt_gemv_fused(self.weights[name], M, K, x[0], threshold, y[0], self.spaces[name])
        else:
            spqt.spqt_gemv_fused_rows(self.weights[name], M, K, x, threshold, y, self.spaces[name])
        return y

    def rotate(self, x):
        """Rotary positions of x [rows, heads, head_dim], in place."""
        rows = torch.arange(self.position, self.position + x.shape[0], device="cuda")
        angles = rows[:, None, None] * self.frequencies
        a, b = x[..., 0::2].float(), x[..., 1::2].float()
        x[..., 0::2], x[..., 1::2] = a * angles.cos() - b * angles.sin(), a * angles.sin() + b * angles.cos()

    def __call__(self, x):
        """x fp16 [rows, hidden] of the next 1 to 4 tokens -> what the layer's attention adds to them."""
        rows = x.shape[0]
        qkv = self.project("qkv", x, self.threshold).view(rows, -1, self.head_dim)
        self.rotate(qkv[:, : self.q_heads + self.kv_heads])
        q, k, v = qkv[None].split([self.q_heads, self.kv_heads, self.kv_heads], dim=2)
        self.lengths += rows                       # (a model does this once for all its layers)
        self.in_cache += rows
        self.position += rows
        spqt.spqt_kv_append(self.codes, self.scales, self.tail, self.table, self.lengths, k, v, weights=self.seen)
        out = torch.empty((1, rows, self.q_heads, self.head_dim), dtype=torch.float16, device="cuda")
        lse = torch.empty((1, rows, self.q_heads), device="cuda")
        spqt.spqt_kv_attention(self.codes, self.scales, self.table, self.lengths, q, out, self.space, lse=lse, weights=self.seen)
        self.last = (q, out)
        if self.in_cache >= self.budget + 64:
            self.evict()
        return self.project("o", out.view(rows, -1), 0.0)

    def evict(self):
        spqt.spqt_kv_evict(self.codes, self.scales, self.tail, self.seen, self.table, self.lengths, self.budget, self.recent, self.spare, self.new_lengths, self.kept,
                           exact=True)              # what stays is moved again and again
        self.table, self.spare = self.spare, self.table
        self.lengths, self.new_lengths = self.new_lengths, self.lengths
        self.in_cache = self.budget
        self.evictions += 1

    def cached(self):
        """Keys and values as they stand in the cache, fp16 [tokens, kv heads, head_dim]."""
        k, v = (torch.empty((1, self.in_cache, self.kv_heads, self.head_dim), dtype=torch.float16, device="cuda") for _ in range(2))
        spqt.spqt_kv_read(self.codes, self.scales, self.table, self.lengths, k, v)
        return k[0], v[0]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("hidden", 4096), ("q-heads", 32), ("kv-heads", 8), ("head-dim", 128), ("prompt", 500), ("steps", 300), ("budget", 512), ("recent", 64)):
        p.add_argument("--" + name, type=int, default=default)
    p.add_argument("--sparsity", type=float, default=0.5)
    a = p.parse_args(argv)
    layer = Layer(a.hidden, a.q_heads, a.kv_heads, a.head_dim, a.budget, a.recent, a.sparsity)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.prompt, a.hidden), device="cuda", generator=gen).half()
    for first in range(0, a.prompt, 4):
        y = layer(x[first : first + 4].contiguous())[-1:]
    torch.cuda.synchronize()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(a.steps):
        # the next token's hidden state: the rest of the model is a rotation and a normalization here
        x = (y.roll(7, dims=1).float() + torch.randn((1, a.hidden), device="cuda", generator=gen)).half()
        x = (x.float() / x.float().pow(2).mean().sqrt()).half()
        y = layer(x)
    end.record()
    torch.cuda.synchronize()
    per_step = begin.elapsed_time(end) / max(1, a.steps) * 1e3
    print(f"{a.prompt} tokens of prompt, {a.steps} steps of {per_step:.0f} us, {layer.position} positions, {layer.in_cache} in the cache after {layer.evictions} evictions")
    return layer


if __name__ == "__main__":
    main()
