"""The norm over all gradients and clipping against plain sums in 64 bits: mixtures of types, odd sizes, views, many tensors, values of any size, in place and
not, streams, graphs."""
import math

import pytest
import torch

from operator_util import DTYPES, U32, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(shape, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * std).to(dtype).to(DEV)


def norm64(grads):
    return math.sqrt(math.fsum(float((g.cpu().double() ** 2).sum()) for g in grads))


def check(grads, clipped, norm, max_norm, eps=1e-6):
    """norm: squares and sums of 64 bits, one rounding to fp32.  factor: norm's rounding, a sum, a quotient; a product and the rounding to the type then."""
    want = norm64(grads)
    assert norm.dtype == torch.float32 and norm.dim() == 0
    assert abs(float(norm) - want) <= 1.01 * U32 * want + 2.0 ** -150
    factor = min(1.0, max_norm / (want + eps))
    for i, (g, c) in enumerate(zip(grads, clipped)):
        assert c.shape == g.shape and c.dtype == g.dtype
        ref = g.cpu().double() * factor
        assert_within(c, ref, 5 * U32 * ref.abs(), i)


SHAPES = {
    "one_value": [(1,)],
    "few": [(7,), (3, 5), (2, 3, 4)],
    "odd": [(1001,), (33, 77), (4099,), (1,), (8191,)],
    "layer": [(8, 128, 256), (8, 128, 256), (8, 256, 128), (128, 8), (128,), (128,)],
    "empty_among": [(0,), (5, 0, 3), (12,), (0,)],
    "only_empty": [(0,), (0, 4)],
    "many": [(i % 37 + 1, i % 11 + 1) for i in range(150)],
    "large": [(4096, 4100), (3,), (2049, 1025)],
    "just_a_launch": [(17,)] * 48,
    "one_more": [(17,)] * 49,
}


@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "mixed"])
@pytest.mark.parametrize("name", SHAPES)
def test_norm_and_clipping(name, dtype, max_norm):
    from paper_2508_18376_amd import moe_clip_grads, moe_grad_norm
    types = list(DTYPES.values()) if dtype == "mixed" else [DTYPES[dtype]]
    grads = [make(s, types[i % len(types)], i) for i, s in enumerate(SHAPES[name])]
    print(name, dtype, max_norm, flush=True)
    clipped, norm = moe_clip_grads(grads, max_norm)
    torch.cuda.synchronize()
    check(grads, clipped, norm, max_norm)
    assert torch.equal(moe_grad_norm(grads), norm)
    mine = [g.clone() for g in grads]
    again, same = moe_clip_grads(mine, max_norm, out=mine)
    assert torch.equal(norm, same) and all(a.data_ptr() == m.data_ptr() for a, m in zip(again, mine))
    assert all(torch.equal(a, c) for a, c in zip(mine, clipped))
    outs = [torch.full_like(g, 7.0) for g in grads]
    got, _ = moe_clip_grads(tuple(grads), max_norm, out=outs)
    assert got is outs and all(torch.equal(a, c) for a, c in zip(outs, clipped))


def test_views():
    """Rows of a wider tensor, both halves of one, transposed and permuted ones, a column's values of one each, in and out of other layouts than each other."""
    from paper_2508_18376_amd import moe_clip_grads
    wide = make((3, 40, 150), torch.bfloat16, 1)
    base = make((64, 48), torch.float32, 2)
    grads = [wide[:, :, :70], wide[:, :, 70:141], base.t(), make((4, 5, 6), torch.float16, 3).permute(2, 0, 1), make((30, 1), torch.float32, 4)[::2, 0][:1],
             make((9, 20), torch.bfloat16, 5)[2:7, 3:], make((1000,), torch.bfloat16, 6)[1:]]
    clipped, norm = moe_clip_grads(grads, 1.0)
    check(grads, clipped, norm, 1.0)
    keep, kept = wide.clone(), [g.clone() for g in grads]
    moe_clip_grads(grads, 1.0, out=grads)
    check(kept, grads, norm, 1.0)
    assert all(torch.equal(g, c) for g, c in zip(grads, clipped))
    assert torch.equal(wide[:, :, 141:], keep[:, :, 141:])
    rows = make((33, 50), torch.float32, 7)
    out = [torch.full((33, 64), 7.0, device=DEV)[:, 5:55]]
    got, norm = moe_clip_grads([rows], 1.0, out=out)
    check([rows], got, norm, 1.0)
    assert (out[0]._base[:, :5] == 7).all() and (out[0]._base[:, 55:] == 7).all()


@pytest.mark.parametrize("dtype,size", [("f32", 1e25), ("f32", 1e-30), ("bf16", 1e30), ("bf16", 1e-35), ("f16", 6e4), ("f16", 1e-7), ("f32", 1e38)])
def test_squares_beyond_fp32(dtype, size):
    """Values whose squares are infinite or zero in fp32: the norm is right where it is an fp32 number."""
    from paper_2508_18376_amd import moe_clip_grads
    g = [torch.full((3,), size, device=DEV).to(DTYPES[dtype]), torch.full((5,), -size / 2, device=DEV).to(DTYPES[dtype])]
    clipped, norm = moe_clip_grads(g, size / 4, eps=0.0)
    check(g, clipped, norm, size / 4, 0.0)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_values_that_are_not_finite_show(bad):
    from paper_2508_18376_amd import moe_clip_grads
    grads = [torch.ones(100, device=DEV), torch.ones(50, 3, device=DEV, dtype=torch.bfloat16)]
    grads[1][7, 1] = bad
    clipped, norm = moe_clip_grads(grads, 1.0)
    if math.isnan(bad):
        assert torch.isnan(norm) and all(torch.isnan(c).all() for c in clipped)
    else:
        assert torch.isinf(norm) and (clipped[0] == 0).all() and torch.isnan(clipped[1][7, 1]) and int(torch.isnan(clipped[1]).sum()) == 1


def test_zeros():
    from paper_2508_18376_amd import moe_clip_grads
    grads = [torch.zeros(100, device=DEV), torch.zeros(3, device=DEV)]
    clipped, norm = moe_clip_grads(grads, 1.0)
    assert float(norm) == 0 and all((c == 0).all() for c in clipped)
    clipped, norm = moe_clip_grads(grads, 0.0, eps=0.0)  # 0 / 0: as the formula says
    assert float(norm) == 0 and all(torch.isnan(c).all() for c in clipped)


def test_the_same_tensor_twice():
    """Counts twice; written to two places, but not in place."""
    from paper_2508_18376_amd import DsmoeError, moe_clip_grads
    g = make((1000,), torch.float32, 8)
    clipped, norm = moe_clip_grads([g, g], 1.0)
    check([g, g], clipped, norm, 1.0)
    with pytest.raises(DsmoeError, match="twice"):
        moe_clip_grads([g, g], 1.0, out=[g, g])


def test_more_values_than_32_bits_count():
    """One tensor of more than 2^32 bytes and 2^31 values: its last values count and are clipped."""
    from paper_2508_18376_amd import moe_clip_grads
    n = (1 << 31) + 4099
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g[0], g[n - 1], g[1 << 31] = 3.0, 4.0, 12.0
    out, norm = moe_clip_grads([g], 6.5, eps=0.0, out=[g])
    assert float(norm) == 13.0
    torch.cuda.synchronize()
    assert (float(g[0]), float(g[n - 1]), float(g[1 << 31]), float(g[5])) == (1.5, 2.0, 6.0, 0.0)
    del g, out
    torch.cuda.empty_cache()


def test_other_stream_and_graph():
    """Replayed with other values, and between replays of another graph and eager calls of the same tensors."""
    from paper_2508_18376_amd import moe_clip_grads, moe_grad_norm
    a, b = make((300, 70), torch.bfloat16, 9), make((5001,), torch.float32, 10)
    want, norm = moe_clip_grads([a, b], 2.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, same = moe_clip_grads([a, b], 2.0, stream=side)
    other = moe_grad_norm([a, b], stream=side)
    side.synchronize()
    assert torch.equal(same, norm) and torch.equal(other, norm) and all(torch.equal(x, y) for x, y in zip(got, want))
    sa, sb = torch.zeros_like(a), torch.zeros_like(b)
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        clipped, n1 = moe_clip_grads([sa, sb], 2.0)
    with torch.cuda.graph(two):
        n2 = moe_grad_norm([sb, sa])
    for i in range(3):
        scale = 1.0 if i != 1 else 0.001
        sa.copy_(a * scale)
        sb.copy_(b * scale)
        one.replay()
        two.replay()
        torch.cuda.synchronize()
        eager, n = moe_clip_grads([sa, sb], 2.0)
        assert torch.equal(n1, n) and all(torch.equal(x, y) for x, y in zip(clipped, eager))
        assert abs(float(n2) - float(n)) <= 2.5 * U32 * float(n)  # (another order of the tensors)


def test_values_that_a_graph_kept_are_not_overwritten_in_silence():
    from paper_2508_18376_amd import moe_clip_grads
    leaf, g = torch.ones(24, device=DEV, requires_grad=True), torch.ones(24, device=DEV)
    loss = (leaf * g).sum()
    moe_clip_grads([g], 1.0, out=[g])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
