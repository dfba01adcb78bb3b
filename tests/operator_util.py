"""Shared by the tests of the operators beside the layer: plain implementations in 64 bits and the bounds on what fp32 sums and one rounding to
the output's type may be off by."""
from __future__ import annotations

import torch

U32 = 2.0 ** -24  # half a step of fp32, relative
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_SUBNORMAL = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_within(got, ref, err, what):
    """got (rounded once to its type) against ref (64 bits), where the value before the rounding may be off by err."""
    got64 = got.detach().cpu().double()
    assert got64.shape == ref.shape, (what, got64.shape, ref.shape)
    bound = err + half_step(got.dtype) * (ref.abs() + err) + HALF_SUBNORMAL[got.dtype]
    over = (got64 - ref).abs() - bound
    assert not torch.isnan(got64).any(), what
    if over.numel():
        worst = over.argmax()
        assert over.max() <= 0, (what, float(got64.flatten()[worst]), float(ref.flatten()[worst]), float(bound.flatten()[worst]), int((over > 0).sum()))


def same_bits(a, b):
    """Equal, NaN in the same places."""
    t = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.view(t), b.view(t))


def spans(offsets, rows):
    """[lo, hi) of each group as the calls define them for any table: clamped to the rows, and to the largest offset before."""
    at, out = 0, []
    bounds = [min(max(int(o), 0), rows) for o in offsets]
    at = bounds[0]
    for b in bounds[1:]:
        hi = max(at, b)
        out.append((at, hi))
        at = hi
    return out


def grouped_reference(x, w, offsets, transposed=False):
    """(y, sum of the products' magnitudes) in 64 bits on the CPU."""
    x64, w64 = x.cpu().double(), w.cpu().double()
    y = torch.zeros(x.shape[0], w.shape[1 if transposed else 2], dtype=torch.float64)
    mag = torch.zeros_like(y)
    for g, (lo, hi) in enumerate(spans(offsets.tolist(), x.shape[0])):
        m = w64[g].t() if transposed else w64[g]
        y[lo:hi], mag[lo:hi] = x64[lo:hi] @ m, x64[lo:hi].abs() @ m.abs()
    return y, mag


def grouped_dw_reference(x, dy, offsets):
    x64, d64 = x.cpu().double(), dy.cpu().double()
    at = spans(offsets.tolist(), x.shape[0])
    dw = torch.stack([x64[lo:hi].t() @ d64[lo:hi] for lo, hi in at])
    return dw, torch.stack([x64[lo:hi].abs().t() @ d64[lo:hi].abs() for lo, hi in at])


def product_error(mag, terms):
    """A sum of `terms` products in fp32, in any order: (terms + 1) half steps of the sum of magnitudes at most; twice that, because the
    matrix instructions may cut bits off where they add up inside."""
    return 2 * (terms + 2) * U32 * mag


def offsets_of(counts, first=0):
    return torch.tensor([first] + [first + sum(counts[:i + 1]) for i in range(len(counts))], dtype=torch.int32)
