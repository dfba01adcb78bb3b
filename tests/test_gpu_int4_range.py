"""Products with weights in 4 bits at the ends of the range, in every kernel: infinities in x, values of x and scales whose sums taken apart are beyond fp32 though the
products are not."""
import pytest
import torch

from int4_single_util import on_16_bytes
from int4_util import random_weights, reference, unpacked
from operator_util import DTYPES, assert_within, offsets_of
from test_gpu_int4_matmul import call, make

pytestmark = pytest.mark.gpu

# rows of each group, k, n: registers; the same without alignment; tiles of 16, 32 and 64 rows, in parts and not; tiles of few rows for one group of many; tiles of many
# rows; the plain path
SHAPES = {
    "one_row": ([1], 520, 136),
    "sixteen": ([16], 512, 136),
    "odd_few": ([9, 3], 203, 77),
    "two_sixteens": ([30, 20], 203, 77),
    "tiles_of_16_parts": ([3], 8200, 136),
    "tiles_of_32_parts": ([20], 8192, 136),
    "tiles_of_32_several": ([i % 40 for i in range(24)], 328, 520),
    "tiles_of_64": ([40, 70], 264, 520),
    "one_group": ([300], 512, 136),
    "tiles_of_many": ([2100, 2100], 264, 2008),
    "plain": ([100, 70], 203, 77),
}


def on_gpu(w, k):
    """Rows on 16 bytes where the other sizes let the fast paths take them."""
    return on_16_bytes(w.to("cuda")) if k % 8 == 0 else w


@pytest.mark.parametrize("block", [32, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", SHAPES)
def test_infinities_in_x(name, dtype, block):
    """An infinity times a weight is one of the weight's sign, NaN where the weight is zero; two of different signs are NaN.  The other rows do not notice."""
    counts, k, n = SHAPES[name]
    dt, off, R = DTYPES[dtype], offsets_of(counts, 0), sum(counts)
    x = make((R, k), dt, 41)
    w, scale, zero = random_weights(len(counts), n, k, block, dt, block == 32, 42)
    _, err = reference(x, w, scale, zero, off, block)
    inf = float("inf")
    x[0, k // 2] = inf
    x[R // 2, k - 1] = -inf if R > 1 else inf
    if R > 2:
        x[R - 1, 0], x[R - 1, k - 2] = inf, -inf
    y = call(x, on_gpu(w, k), scale, zero, off, block).cpu()
    q, z, s = unpacked(w, scale, zero, k, block)
    ref, at = torch.zeros(R, n, dtype=torch.float64), 0
    for g, rows in enumerate(counts):
        ref[at:at + rows] = x[at:at + rows].double() @ ((q[g] - z[g]) * s[g]).t()
        at += rows
    assert torch.isinf(ref).any() and torch.equal(torch.isnan(y), torch.isnan(ref))
    assert torch.equal(torch.isinf(y), torch.isinf(ref)) and torch.equal(y[torch.isinf(ref)].double(), ref[torch.isinf(ref)])
    good = torch.isfinite(ref)
    assert_within(torch.where(good, y, 0), torch.where(good, ref, 0.0), torch.where(good, err, 0.0), "y")


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("name", SHAPES)
def test_sums_of_x_beyond_fp32(name, wide):
    """Values up to the largest bf16 number with weights that bring the results back."""
    counts, k, n = SHAPES[name]
    off, R = offsets_of(counts, 0), sum(counts)
    x = (torch.rand(R, k, generator=torch.Generator().manual_seed(43)) * 2 - 1).mul(3.38e38).bfloat16()
    x[:, ::2] = x[:, ::2].abs()
    w, scale, zero = random_weights(len(counts), n, k, 64, torch.float32 if wide else torch.bfloat16, True, 44)
    scale = (scale.double() * 1e-9).to(scale.dtype)
    y = call(x, on_gpu(w, k), scale, zero, off, 64)
    assert_within(y, *reference(x, w, scale, zero, off, 64), "y")


@pytest.mark.parametrize("name", SHAPES)
def test_scales_whose_sums_are_beyond_fp32(name):
    """Weights of s, -s and a few zeros that nearly cancel, with s so large that a block's sum of x s is beyond fp32 (32 s), and a few products are not.
    All of it is whole sixteenths of s, so that the results have no error."""
    counts, k, n = SHAPES[name]
    off, R, G = offsets_of(counts, 0), sum(counts), len(counts)
    gen = torch.Generator().manual_seed(45)
    q = torch.where(torch.arange(2 * ((k + 1) // 2)) % 2 == 0, 9, 7).repeat(G, n, 1).to(torch.uint8)
    q.scatter_(2, torch.randint(0, k, (G, n, 3), generator=gen), 8)
    w = q[:, :, 0::2] | q[:, :, 1::2] << 4
    scale = torch.full((G, n, -(-k // 32)), 2.0 ** 123)
    x = torch.ones(R, k, dtype=torch.bfloat16)
    y = call(x, on_gpu(w, k), scale, None, off, 32)
    ref, _ = reference(x, w, scale, None, off, 32)
    assert torch.equal(y.cpu().double(), ref)
