"""CPU oracle of the prompt side in 8-bit integers.  TEST INFRASTRUCTURE ONLY.

Only the tests may import this module.  torch on the CPU, from the definitions: codes and scales in the fp32 steps that define them, one row after the
other; norms and products in 64 bits, with a bound on what fp32 steps may be off by.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24                       # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def quantize(x):
    """x [rows, K] of any floating type that fp32 holds -> (codes int8, scales fp32)."""
    x = x.float()
    codes, scales = torch.zeros(x.shape, dtype=torch.int8), torch.full((x.shape[0],), float("nan"))
    for r in range(x.shape[0]):
        if not torch.isfinite(x[r]).all():
            continue
        top = torch.clamp(x[r].abs().max(), min=2.0 ** -100)
        scales[r] = top / torch.tensor(127.0)
        codes[r] = torch.round(x[r] * (torch.tensor(127.0) / top)).to(torch.int8)
    return codes, scales


def read(codes, scales, dtype):
    v = codes.float() * scales[:, None]
    largest = torch.finfo(dtype).max
    return torch.where(v.isnan(), v, v.clamp(-largest, largest)).to(dtype)


# How many halves of fp32's steps 1 / sqrt(mean of squares + eps) may be off by, relative: a thread adds at most 64 squares one after the other, 6 + 16
# additions join the threads, and the root halves that; then mean, eps, root and quotient.
RMS_STEPS = (64 + 22) / 2 + 4


def norm(h, gain, block=None, block_gain=None, gate=None, residual=1.0, eps=1e-5, offset=0.0):
    """64-bit tensors -> (s, x, bounds of what fp32 steps make of s and of x, before either is rounded)."""
    K = h.shape[1]

    def normed(v, off, g):
        by = 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + eps)
        x = v * by * (offset + g)
        moved = torch.sqrt((off * off).mean(dim=1, keepdim=True)) * by        # what the root of the mean makes of `off`, relative, at most
        return x, off * by * (offset + g).abs() + x.abs() * (moved + (RMS_STEPS + 4) * U)

    s, off = h, torch.zeros_like(h)
    if block is not None:
        z, off = block, torch.zeros_like(block)
        if block_gain is not None:
            z, off = normed(z, off, block_gain)
        if gate is not None:
            z, off = z * gate, off * gate.abs() + (z * gate).abs() * U
        s = residual * h + z
        off = off + s.abs() * U + (residual * h).abs() * U
    x, far = normed(s, off, gain)
    return s, x, off, far


def product(codes, scales, weights, weight_scales, bias=None, gated=False):
    """(y in 64 bits, bound of what fp32 steps make of it before it is rounded to y's type)."""
    acc = codes.double() @ weights.double().t()                # whole numbers under 2^53: exact
    v = acc * scales.double()[:, None] * weight_scales.double()
    off = 3 * U * v.abs()
    if bias is not None:
        v = v + bias.double()
        off = off + U * v.abs()
    off = off * 1.0001 + 1e-38
    if not gated:
        return v, off
    F = v.shape[1] // 2
    g, u, dg, du = v[:, :F], v[:, F:], off[:, :F], off[:, F:]
    y = g * torch.sigmoid(g) * u
    # silu' is at most 1.1; exp(-g) is off by |g| of fp32's steps and a few, and 1 + exp(-g), quotient and product by a half each
    return y, 1.1 * dg * u.abs() + (g * torch.sigmoid(g)).abs() * du + y.abs() * (2 * g.abs() + 16) * U + 1e-36
