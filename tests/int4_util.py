"""Products with weights in 4 bits in 64 bits on the CPU, with bounds on what the operator may be off by."""
from __future__ import annotations

import torch

from operator_util import half_step, product_error, spans


def random_weights(G, n, k, block, dtype_of_scale, zeros, seed, most_zero=15):
    """(w, w_scale, w_zero or None): any 4-bit numbers, scales of both signs over two decades."""
    gen = torch.Generator().manual_seed(seed)
    B = -(-k // block)
    w = torch.randint(0, 256, (G, n, (k + 1) // 2), generator=gen, dtype=torch.uint8)
    scale = (torch.rand(G, n, B, generator=gen) * 4.6 - 4.6).exp() * torch.where(torch.rand(G, n, B, generator=gen) < 0.2, -0.1, 0.1)
    zero = torch.randint(0, most_zero + 1, (G, n, B), generator=gen, dtype=torch.uint8) if zeros else None
    return w, scale.to(dtype_of_scale), zero


def unpacked(w, w_scale, w_zero, k, block):
    """(q, z, s) of each weight, [G][n][k] in 64 bits."""
    q = torch.stack([w & 15, w >> 4], 3).flatten(2)[:, :, :k].double()
    at = torch.arange(k) // block
    z = torch.full_like(q, 8.0) if w_zero is None else w_zero.double()[:, :, at]
    return q, z, w_scale.double()[:, :, at]


def reference(x, w, w_scale, w_zero, offsets, block):
    """(y, bound before the rounding of the result) in 64 bits.

    16-bit types: a weight (q - z) s may be rounded to x's type (f16: where that is subnormal next to the channel's largest scale, to 2^-25 of it), after a
    difference and a product in fp32; or it is taken apart, 16 (1 + q / 16) s - (16 + z) s, whose sums are larger than the weights'.  fp32: neither."""
    x64, k = x.cpu().double(), x.shape[1]
    q, z, s = unpacked(w.cpu(), w_scale.cpu(), None if w_zero is None else w_zero.cpu(), k, block)
    R = x.shape[0]
    y, err = torch.zeros(R, w.shape[1], dtype=torch.float64), torch.zeros(R, w.shape[1], dtype=torch.float64)
    for g, (lo, hi) in enumerate([(0, R)] if offsets is None else spans(offsets.tolist(), R)):
        if hi == lo:
            continue
        xg = x64[lo:hi]
        weight = (q[g] - z[g]) * s[g]
        mag = xg.abs() @ weight.abs().t()
        y[lo:hi] = xg @ weight.t()
        if x.dtype == torch.float32:
            err[lo:hi] = product_error(mag, k + 4)
            continue
        apart = xg.abs() @ ((32 + q[g] + z[g]) * s[g].abs()).t()
        err[lo:hi] = half_step(x.dtype) * mag + product_error(apart, k + 8)
        if x.dtype == torch.float16:
            err[lo:hi] += 2.0 ** -25 * xg.abs().sum(1, keepdim=True) * 2 * s[g].abs().amax(1)
    return y, err
