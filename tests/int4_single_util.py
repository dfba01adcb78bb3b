"""Rows of x with a single value: what a product with weights in 4 bits then gives is one weight times that value, so that the weight itself, its block's scale and zero
point, and whether the value was seen at all can be checked, which the bounds of long sums hide."""
from __future__ import annotations

import torch

from int4_util import unpacked
from operator_util import U32, assert_within, half_step, spans


def places(k):
    """Where the values are: the ends, both sides of each 128 values (a stage, a step, and whatever parts are made of them), and one inside."""
    gen = torch.Generator().manual_seed(k)
    at = {0, k - 1, max(k - 2, 0), max(k - 8, 0), max(k - 9, 0), max(k - 32, 0), max(k - 33, 0)}
    for b in range(0, k, 128):
        at |= {b, max(b - 1, 0), min(b + int(torch.randint(0, 128, (1,), generator=gen)), k - 1)}
    return sorted(at, key=lambda p: (p * 7919) % 104729)  # (in no order, so that neighbouring rows are apart)


def rows_of(at, k, dtype, seed):
    """x, a row for each of the places `at`, and its values: of both signs, from 1 to 2, with all of the type's bits."""
    gen = torch.Generator().manual_seed(seed)
    v = ((1 + torch.rand(len(at), generator=gen)) * torch.where(torch.rand(len(at), generator=gen) < 0.5, -1.0, 1.0)).to(dtype)
    x = torch.zeros(len(at), k, dtype=dtype)
    x[torch.arange(len(at)), torch.tensor(at)] = v
    return x, v


def on_16_bytes(w):
    """w with rows that start on 16 bytes, as a view into a tensor whose other bytes are not zero."""
    row = w.shape[2]
    wide = torch.full((*w.shape[:2], -(-row // 16) * 16), 0xa7, dtype=torch.uint8, device=w.device)
    wide[:, :, :row] = w
    return wide[:, :, :row]


def products(at, v, w, w_scale, w_zero, offsets, k, block, rounded=False):
    """(y, bound): the weight is not rounded.  The two sums that it is taken apart into are of one value each: rounded are the scale times the zero point, both
    products and their sum, four half steps, which count twice (the matrix instructions may cut off).
    rounded: it is, to x's type, once (f16: or to 2^-25 of twice the channel's largest scale, where it is subnormal next to that)."""
    q, z, s = unpacked(w, w_scale, w_zero, k, block)
    y, err = torch.zeros(len(at), w.shape[1], dtype=torch.float64), torch.zeros(len(at), w.shape[1], dtype=torch.float64)
    for g, (lo, hi) in enumerate(spans(offsets.tolist(), len(at))):
        p, x = torch.tensor(at[lo:hi], dtype=torch.long), v[lo:hi, None].double()
        y[lo:hi] = x * ((q[g] - z[g]) * s[g])[:, p].t()
        err[lo:hi] = 8 * U32 * x.abs() * ((32 + q[g] + z[g]) * s[g].abs())[:, p].t()
        if rounded:
            err[lo:hi] += half_step(v.dtype) * y[lo:hi].abs()
            if v.dtype == torch.float16:
                err[lo:hi] += 2.0 ** -25 * x.abs() * 2 * s[g].abs().amax(1)
    return y, err


def check(y, *how, **kw):
    assert_within(y, *products(*how, **kw), "y")
