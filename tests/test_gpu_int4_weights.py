"""Products with weights in 4 bits, weight by weight: no value, block, stage or part is lost, and of few rows nothing but the result is rounded."""
import pytest
import torch

from int4_single_util import check, on_16_bytes, places, rows_of
from int4_util import random_weights, reference
from operator_util import DTYPES, assert_within, offsets_of
from test_gpu_int4_matmul import SHAPES as OTHERS, call, make
from test_gpu_int4_sizes import SHAPES as SIZES

pytestmark = pytest.mark.gpu

# rows of each group, k, n, whether the weights' rows start on 16 bytes, whether weights are rounded.  Contractions that end inside a stage, with other bytes behind.
SHAPES = {
    "registers_one_row": ([1], 1032, 136, True, False),
    "registers_sixteen": ([16], 4096, 72, True, False),
    "registers_odd": ([9, 3], 1003, 77, False, False),
    "registers_odd_32": ([30, 20], 1203, 77, False, False),
    "tiles_of_16_parts": ([3], 8200, 136, True, False),
    "tiles_of_16_long": ([5], 14344, 72, True, False),
    "tiles_of_16_many": ([i % 9 for i in range(64)], 4104, 520, True, False),
    "tiles_of_32_parts": ([20], 8200, 136, True, False),
    "tiles_of_32_several": ([i % 40 for i in range(24)], 1064, 520, True, False),
    "tiles_of_64": ([40, 70], 2056, 520, True, False),
    "tiles_of_64_one_stage": ([64, 63, 65], 40, 264, True, False),
    "tiles_of_64_blocks": ([50, 30, 20, 10], 200, 264, True, False),
    "one_group": ([300], 4104, 136, True, False),
    "tiles_of_many": ([2100, 2101], 264, 2008, True, True),
    "tiles_of_many_parts": ([4100, 4201], 1096, 1808, True, True),
    "tiles_of_many_halves": ([8300], 136, 1808, True, True),
    "tiles_of_many_short": ([5000, 3300], 8, 1808, True, True),
    "plain": ([100, 70], 1003, 77, False, True),
    "plain_aligned": ([100, 70], 1000, 136, False, True),
}


@pytest.mark.parametrize("block", [32, 64, 128, 4096])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", SHAPES)
def test_each_weight(name, dtype, block):
    counts, k, n, aligned, rounded = SHAPES[name]
    dt, off, R = DTYPES[dtype], offsets_of(counts), sum(counts)
    w, scale, zero = random_weights(len(counts), n, k, block, torch.float32 if block in (32, 4096) else dt, block != 64, 51)
    on_gpu = on_16_bytes(w.to("cuda")) if aligned else w
    print(name, dtype, block, flush=True)
    every = places(k)
    for i in range(0, len(every), R):
        at = ((every[i:] + every) * (R // len(every) + 1))[:R]
        x, v = rows_of(at, k, dt, 52 + i)
        check(call(x, on_gpu, scale, zero, off, block), at, v, w, scale, zero, off, k, block, rounded=rounded)


ALIGNED = {name: s for name, s in dict(OTHERS, **SIZES).items() if s[3] % 8 == 0 and s[3] % 32 and s[4] % 8 == 0}


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", ALIGNED)
def test_whole_sums_on_16_bytes(name, dtype, block):
    """The sizes at which kernels, tiles and cuts change, in the layout that the fast paths take, where the weights' rows have other bytes behind them."""
    counts, before, after, k, n = ALIGNED[name]
    dt, off = DTYPES[dtype], offsets_of(counts, before)
    R = before + sum(counts) + after
    x = make((R, k), dt, 53)
    w, scale, zero = random_weights(len(counts), n, k, block, torch.float32 if block == 32 else dt, block != 64, 54)
    fast = on_16_bytes(w.to("cuda"))
    print(name, dtype, block, flush=True)
    y = call(x, fast, scale, zero, off, block)
    assert_within(y, *reference(x, w, scale, zero, off, block), "y")
    held = torch.zeros(R, dtype=torch.bool)
    held[before:before + sum(counts)] = True
    assert (y.cpu()[~held] == 0).all()
    assert torch.equal(y, call(x, fast, scale, zero, off, block))
