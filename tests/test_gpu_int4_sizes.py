"""Products with weights in 4 bits at the sizes where another kernel, another tile or another cut takes over: few rows in many groups, hundreds of rows in many
groups, more tiles than compute units with a few left over, which are halved or cut along the contraction; and at these, foreign values, strides, graphs, weights
of any size and rows beyond 2^32 bytes."""
import pytest
import torch

from int4_util import random_weights, reference
from operator_util import DTYPES, assert_within, offsets_of, same_bits
from test_gpu_int4_matmul import DEV, call, make

pytestmark = pytest.mark.gpu

# counts of the groups, rows in front of the first and behind the last one, k, n
SHAPES = {
    "few_rows_of_many": ([i % 4 for i in range(64)], 0, 3, 328, 520),
    "few_rows_long_sums": ([i % 4 for i in range(64)], 1, 0, 2064, 520),
    "sixteens_of_many": ([9 + i % 13 for i in range(40)], 0, 2, 264, 520),
    "sixteens_long_sums": ([9 + i % 13 for i in range(20)], 0, 2, 2120, 1032),
    "sixties": ([30 + i % 90 for i in range(20)], 2, 0, 1104, 600),
    "hundreds": ([200 + i % 7 for i in range(40)], 0, 5, 136, 392),
    "hundreds_parts": ([257] * 18, 0, 0, 1104, 1160),
    "halves": ([5000, 0, 3300], 0, 0, 136, 1808),
    "halves_odd": ([8300 - 40, 40], 0, 0, 264, 2040),
    "parts": ([8200, 100], 0, 0, 2048, 1808),
    "empty_but_one": ([0, 0, 9000, 0], 100, 60, 200, 1040),
}


@pytest.mark.parametrize("block", [32, 64, 128, 4096])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", SHAPES)
def test_products(name, dtype, block):
    counts, before, after, k, n = SHAPES[name]
    dt, off = DTYPES[dtype], offsets_of(counts, before)
    R, G = before + sum(counts) + after, len(counts)
    zeros, wide = block != 64, block in (32, 4096)
    x = make((R, k), dt, 21)
    w, scale, zero = random_weights(G, n, k, block, torch.float32 if wide else dt, zeros, 22)
    print(name, dtype, block, R, G, k, n, flush=True)
    y = call(x, w, scale, zero, off, block)
    assert_within(y, *reference(x, w, scale, zero, off, block), "y")
    held = torch.zeros(R, dtype=torch.bool)
    held[before:before + sum(counts)] = True
    assert (y.cpu()[~held] == 0).all()
    assert torch.equal(y, call(x, w, scale, zero, off, block))


@pytest.mark.parametrize("k", [136, 2048])
def test_one_group_without_a_table(k):
    x = make((8300, k), torch.bfloat16, 23)
    w, scale, zero = random_weights(1, 1808, k, 128, torch.bfloat16, True, 24, most_zero=255)
    y = call(x, w, scale, zero, None, 128)
    assert_within(y, *reference(x, w, scale, zero, None, 128), "y")
    assert torch.equal(y, call(x, w, scale, zero, offsets_of([8300]), 128))


# groups, rows of each, k, n: the tiles of few rows, and those of many
BOTH = {"few": (3, 150, 264, 520), "many": (2, 2100, 264, 2008)}


@pytest.mark.parametrize("size", BOTH)
@pytest.mark.parametrize("block", [32, 128])
def test_other_rows_and_groups_values_do_not_leak(size, block):
    G, rows, k, n = BOTH[size]
    off = offsets_of([rows] * G, 2)
    R = G * rows + 5
    x = make((R, k), torch.bfloat16, 25)
    w, scale, zero = random_weights(G, n, k, block, torch.float32, True, 26)
    ref, err = reference(x, w, scale, zero, off, block)
    x[:2], x[-3:], x[3] = float("nan"), float("inf"), float("nan")
    x[4, k // 2] = float("inf")
    scale[1, 7, 0], scale[1, 9, -1] = float("nan"), float("inf")
    y = call(x, w, scale, zero, off, block).cpu()
    assert (y[:2] == 0).all() and (y[-3:] == 0).all() and torch.isnan(y[3]).all() and not torch.isfinite(y[4]).any()
    good = torch.ones(R, n, dtype=torch.bool)
    good[3:5] = False
    good[2 + rows:2 + 2 * rows, [7, 9]] = False
    assert not torch.isfinite(y[2 + rows:2 + 2 * rows, [7, 9]]).any()
    assert_within(torch.where(good, y, 0), torch.where(good, ref, 0.0), torch.where(good, err, 0.0), "y")


@pytest.mark.parametrize("size", BOTH)
def test_strided_and_overlapping(size):
    """All operands inside wider tensors, then strides of zero for the weights of all groups and channels."""
    from paper_2508_18376_amd import moe_int4_matmul
    G, rows, k, n = BOTH[size]
    dt, block, R = torch.float16, 64, G * rows
    off, B = offsets_of([rows] * G), -(-k // 64)
    x = make((R, k + 24), dt, 27)
    w, scale, zero = random_weights(G, n + 1, 2 * (-(-k // 32) * 16 + 48), block, dt, True, 28)
    xd, wd, sd, zd = x.to(DEV)[:, 8:8 + k], w.to(DEV)[:, :n, :k // 2], scale.to(DEV)[:, 1:, :B], zero.to(DEV)[:, 1:, 1:B + 1]
    wide = torch.full((R, n + 16), 7.0, dtype=dt, device=DEV)
    moe_int4_matmul(xd, wd, sd, zd, off.to(DEV), block=block, out=wide[:, 8:8 + n])
    assert_within(wide[:, 8:8 + n], *reference(xd, wd.contiguous(), sd.contiguous(), zd.contiguous(), off, block), "y")
    assert (wide[:, :8] == 7).all() and (wide[:, 8 + n:] == 7).all()
    wd, sd, zd = wd[:1, :1].contiguous().expand(G, n, -1), sd[:1, :1].contiguous().expand(G, n, -1), zd[:1, :1].contiguous().expand(G, n, -1)
    y = moe_int4_matmul(xd, wd, sd, zd, off.to(DEV), block=block)
    assert_within(y, *reference(xd, wd, sd, zd, off, block), "y")


@pytest.mark.parametrize("scale_of", [1e-7, 1e-4, 30.0])
@pytest.mark.parametrize("size", BOTH)
def test_half_precision_weights_of_any_size(size, scale_of):
    G, rows, k, n = BOTH[size]
    off = offsets_of([rows] * G)
    x = make((G * rows, k), torch.float16, 29, min(1 / scale_of, 2000.0) * 0.05)
    w, scale, zero = random_weights(G, n, k, 64, torch.float32, True, 30)
    scale = scale * scale_of
    scale[:, ::3, 1] *= 2.0 ** -12
    scale[:, 5] = 0
    y = call(x, w, scale, zero, off, 64)
    ref, err = reference(x, w, scale, zero, off, 64)
    fits = ref.abs() + err < 65504
    assert fits.float().mean() > 0.9
    assert_within(torch.where(fits, y.cpu().float(), 0.0).half(), torch.where(fits, ref, 0.0), torch.where(fits, err, 0.0), "y")
    assert (y[:, 5] == 0).all()


@pytest.mark.parametrize("size", ["few_rows_long_sums", "hundreds_parts", "parts"])
def test_graphs_and_two_streams(size):
    """Calls whose parts are joined through a workspace: on two streams at once, and in two graphs replayed in turn with eager calls between."""
    from paper_2508_18376_amd import moe_int4_matmul
    counts, before, after, k, n = SHAPES[size]
    off = offsets_of(counts, before).to(DEV)
    xs = [make((before + sum(counts) + after, k), torch.bfloat16, 31 + i).to(DEV) for i in range(2)]
    w, scale, zero = (t.to(DEV) for t in random_weights(len(counts), n, k, 64, torch.bfloat16, True, 33))
    want = [moe_int4_matmul(x, w, scale, zero, off, block=64) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [moe_int4_matmul(x, w, scale, zero, off, block=64, stream=s) for x, s in zip(xs, streams)]
    torch.cuda.synchronize()
    assert all(same_bits(a, b) for a, b in zip(got, want))
    graphs, held, outs = [], [torch.zeros_like(x) for x in xs], []
    for h in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(moe_int4_matmul(h, w, scale, zero, off, block=64))
    for i in range(3):
        for j in range(2):
            held[j].copy_(xs[(i + j) % 2])
            graphs[j].replay()
        eager = moe_int4_matmul(xs[0], w, scale, zero, off, block=64)
        torch.cuda.synchronize()
        assert same_bits(eager, want[0]) and all(same_bits(outs[j], want[(i + j) % 2]) for j in range(2)), i


@pytest.mark.parametrize("size", [(8, 160, 256, 400), (1, 4000, 256, 2008)])
def test_values_beyond_four_gigabytes(size):
    """Rows of x, y and w of which most lie more than 2^32 bytes behind the first, at the widest strides of the tiles."""
    from paper_2508_18376_amd import moe_int4_matmul
    G, rows, k, n = size
    big = torch.empty(G * rows << 21, dtype=torch.bfloat16, device=DEV).view(G * rows, 1 << 21)
    weights = torch.empty(G * n << 22, dtype=torch.uint8, device=DEV).view(G, n, 1 << 22)
    off = offsets_of([rows] * G)
    x = make((G * rows, k), torch.bfloat16, 34)
    w, scale, zero = random_weights(G, n, k, 64, torch.bfloat16, True, 35)
    big[:, :k] = x.to(DEV)
    weights[:, :, :k // 2] = w.to(DEV)
    y = moe_int4_matmul(big[:, :k], weights[:, :, :k // 2], scale.to(DEV), zero.to(DEV), off.to(DEV), block=64, out=big[:, 1024:1024 + n])
    torch.cuda.synchronize()
    assert_within(y, *reference(x, w, scale, zero, off, 64), "y")
    del big, weights, y
    torch.cuda.empty_cache()
