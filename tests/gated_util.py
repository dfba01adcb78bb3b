"""The gated half of a block in 64 bits on the CPU, with bounds on what the operators' fp32 steps and roundings may be off by."""
from __future__ import annotations

import math

import torch

from operator_util import HALF_SUBNORMAL, U32, half_step, product_error, spans

GELU_C, GELU_A = math.sqrt(2 / math.pi), 0.044715
# The largest |f'| and |f''|: Swish 1.0998 and 0.5, GELU by tanh 1.129 and 0.798
SLOPE, CURVE = 1.13, 0.8
# exp overflows in fp32 at 88.7: from there on f is taken as zero, |a| exp(-|z|) < 1e-36
TINY = 1e-36


def activation(a, kind):
    """f, f' in 64 bits, z and z' (f(a) = a sigmoid(z))."""
    if kind == "silu":
        z, dz = a, torch.ones_like(a)
    else:
        z, dz = 2 * GELU_C * (a + GELU_A * a ** 3), 2 * GELU_C * (1 + 3 * GELU_A * a ** 2)
    s = torch.sigmoid(z)
    return a * s, s + a * s * torch.sigmoid(-z) * dz, z, dz


def activation_errors(a, ea, kind):
    """What fp32 may be off by in f and f', where a is off by up to ea: the slopes' bounds times ea; exp's argument is off by 8 half steps at most (z takes
    five roundings, its constants one each), so exp by 8 |z| of them and its own 4, the quotient and products by 4 more; 1 - s by half a step of 1."""
    f, slope, z, dz = activation(a, kind)
    s = torch.sigmoid(z)
    steps = (8 + 8 * z.abs().clamp_max(1e3)) * U32
    return SLOPE * ea + f.abs() * steps + TINY, CURVE * ea + (s + (a * s * torch.sigmoid(-z) * dz).abs()) * 2 * steps + (a * s * dz).abs().clamp_max(1e3) * 4 * U32 + TINY


def reference(x, w1, w3, offsets, kind, dh=None):
    """{"h", "saved", "dx", "dw1", "dw3"}, each (value, bound before the rounding of the result); offsets None: one group."""
    x64, u64, v64 = (t.cpu().double() for t in (x, w1, w3))
    R, G, k, n = x.shape[0], w1.shape[0], x.shape[1], w1.shape[2]
    at = [(0, R)] if offsets is None else spans(offsets.tolist(), R)
    out = {name: (torch.zeros(*shape, dtype=torch.float64), torch.zeros(*shape, dtype=torch.float64))
           for name, shape in (("h", (R, n)), ("saved", (2, R, n)), ("dx", (R, k)), ("dw1", (G, k, n)), ("dw3", (G, k, n)))}
    for g, (lo, hi) in enumerate(at):
        if hi == lo:
            continue
        xg = x64[lo:hi]
        a, b = xg @ u64[g], xg @ v64[g]
        ea, eb = (product_error(xg.abs() @ w[g].abs(), k) for w in (u64, v64))
        f, slope, _, _ = activation(a, kind)
        ef, es = activation_errors(a, ea, kind)

        def put(name, index, value, err):
            out[name][0][index], out[name][1][index] = value, err

        put("saved", (0, slice(lo, hi)), a, ea)
        put("saved", (1, slice(lo, hi)), b, eb)
        put("h", slice(lo, hi), f * b, b.abs() * ef + f.abs() * eb + ef * eb + 2 * U32 * (f * b).abs())
        if dh is None:
            continue
        d = dh[lo:hi].cpu().double()
        step, least = half_step(x.dtype), HALF_SUBNORMAL[x.dtype]
        da, db = d * b * slope, d * f
        eda = d.abs() * (b.abs() * es + slope.abs() * eb + es * eb) + 4 * U32 * da.abs()
        edb = d.abs() * ef + 2 * U32 * db.abs()
        eda, edb = eda + step * (da.abs() + eda) + least, edb + step * (db.abs() + edb) + least
        dx = da @ u64[g].t() + db @ v64[g].t()
        most = [(v.abs() + e) @ w[g].abs().t() for v, e, w in ((da, eda, u64), (db, edb, v64))]
        put("dx", slice(lo, hi), dx, eda @ u64[g].abs().t() + edb @ v64[g].abs().t() + product_error(most[0] + most[1], 2 * n))
        for name, v, e in (("dw1", da, eda), ("dw3", db, edb)):
            put(name, g, xg.t() @ v, xg.abs().t() @ e + product_error(xg.abs().t() @ (v.abs() + e), hi - lo))
    return out
