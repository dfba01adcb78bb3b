"""Products over groups of rows and their gradients against plain products in 64 bits: types, odd and aligned sizes, ragged, empty and missing
groups, strides, streams, graphs, tables out of order."""
import numpy as np
import pytest
import torch

from operator_util import DTYPES, assert_within, grouped_dw_reference, grouped_reference, offsets_of, product_error

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(shape, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * std).to(dtype)


# counts of the groups, rows in front of the first and behind the last one, k, n
SHAPES = {
    "one_row": ([1], 0, 0, 64, 64),
    "one_value": ([1], 0, 0, 1, 1),
    "few_of_many": ([0, 1, 0, 2, 0, 0, 1, 0], 0, 0, 256, 192),
    "decode": ([1, 0, 2, 1, 0, 3, 0, 1], 0, 0, 512, 384),
    "sixteens": ([16, 17, 15, 32, 33], 0, 0, 320, 264),
    "ragged": ([70, 0, 129, 1, 255], 3, 5, 136, 200),
    "spare_ends": ([5, 300], 17, 41, 64, 328),
    "tiles": ([256, 512, 64], 0, 0, 256, 512),
    "long_k": ([40, 9], 0, 0, 2048, 96),
    "long_rows": ([1500, 700], 0, 0, 72, 136),
    "odd": ([37, 0, 131, 6], 2, 3, 101, 77),
    "odd_k": ([65, 64], 0, 0, 203, 128),
    "odd_n": ([65, 64], 0, 0, 128, 203),
    "even_not_aligned": ([90, 45], 0, 1, 130, 166),
    "no_rows_in_groups": ([0, 0, 0], 4, 9, 64, 72),
    "split_k": ([300, 0, 40, 70], 5, 9, 4096, 264),
    "split_n": ([300, 0, 40, 70], 5, 9, 264, 4096),
    "split_rows": ([5000, 0, 1234], 1, 2, 264, 136),
    "split_last_round": ([4200, 3900], 0, 60, 1024, 2304),
    "many_groups": ([i % 3 for i in range(150)], 1, 0, 64, 40),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
def test_products(name, dtype):
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts, before, after, k, n = SHAPES[name]
    dt = DTYPES[dtype]
    off = offsets_of(counts, before)
    R, G = before + sum(counts) + after, len(counts)
    x, w, dy = make((R, k), dt, 1), make((G, k, n), dt, 2, 0.1), make((R, n), dt, 3)
    xd, wd, dyd, offd = x.to(DEV), w.to(DEV), dy.to(DEV), off.to(DEV)
    print(name, dtype, R, G, k, n, flush=True)
    y = moe_grouped_matmul(xd, wd, offd)
    torch.cuda.synchronize()
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, k), "y")
    dx = moe_grouped_matmul(dyd, wd, offd, w_transposed=True)
    torch.cuda.synchronize()
    ref, mag = grouped_reference(dy, w, off, transposed=True)
    assert_within(dx, ref, product_error(mag, n), "dx")
    dw = moe_grouped_matmul_dw(xd, dyd, offd)
    torch.cuda.synchronize()
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dw, ref, product_error(mag, max(counts + [1])), "dw")
    outside = torch.ones(R, dtype=torch.bool)
    outside[before:before + sum(counts)] = False
    assert (y.cpu()[outside] == 0).all() and (dx.cpu()[outside] == 0).all()
    # the same inputs give the same bits
    assert torch.equal(y, moe_grouped_matmul(xd, wd, offd)) and torch.equal(dw, moe_grouped_matmul_dw(xd, dyd, offd))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [8, 3])
def test_strided_rows(dtype, pad):
    """Inputs inside wider tensors, outputs into wider tensors, whose other values stay."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    dt, k, n = DTYPES[dtype], 96, 160
    counts = [33, 0, 140]
    R, off = sum(counts), offsets_of(counts)
    x, w, dy = make((R, k + pad), dt, 4), make((3, k + 1, n + pad), dt, 5, 0.1), make((R, n + pad), dt, 6)
    xd, wd, dyd, offd = x.to(DEV)[:, :k], w.to(DEV)[:, :k, :n], dy.to(DEV)[:, :n], off.to(DEV)
    wide = torch.full((R, n + pad), 7.0, dtype=dt, device=DEV)
    y = moe_grouped_matmul(xd, wd, offd, out=wide[:, :n])
    ref, mag = grouped_reference(x[:, :k], w[:, :k, :n], off)
    assert_within(y, ref, product_error(mag, k), "y")
    assert (wide[:, n:] == 7).all()
    dx = moe_grouped_matmul(dyd, wd, offd, w_transposed=True)
    ref, mag = grouped_reference(dy[:, :n], w[:, :k, :n], off, transposed=True)
    assert_within(dx, ref, product_error(mag, n), "dx")
    wide = torch.full((3, k + 1, n + pad), 7.0, dtype=dt, device=DEV)
    dw = moe_grouped_matmul_dw(xd, dyd, offd, out=wide[:, :k, :n])
    ref, mag = grouped_dw_reference(x[:, :k], dy[:, :n], off)
    assert_within(dw, ref, product_error(mag, max(counts)), "dw")
    assert (wide[:, k:] == 7).all() and (wide[:, :, n:] == 7).all()


def test_rows_and_weights_that_overlap():
    """Strides of zero: one row for all tokens, one weight for all groups."""
    from paper_2508_18376_amd import moe_grouped_matmul
    off = offsets_of([40, 30])
    x, w = make((1, 64), torch.bfloat16, 7), make((1, 64, 72), torch.bfloat16, 8)
    y = moe_grouped_matmul(x.to(DEV).expand(70, 64), w.to(DEV).expand(2, 64, 72), off.to(DEV))
    ref, mag = grouped_reference(x.expand(70, 64), w.expand(2, 64, 72), off)
    assert_within(y, ref, product_error(mag, 64), "y")


@pytest.mark.parametrize("k", [64, 61])
def test_other_groups_values_do_not_leak(k):
    """NaN and infinities in one group's rows or weights, and in rows of no group, stay out of the other groups' results and gradients."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts, n = [21, 50, 13], 88
    off = offsets_of(counts, 4)
    R = 4 + sum(counts) + 6
    x, w, dy = make((R, k), torch.bfloat16, 9), make((3, k, n), torch.bfloat16, 10), make((R, n), torch.bfloat16, 11)
    for t in (x, dy):
        t[:4], t[-6:], t[25:75] = float("nan"), float("inf"), float("nan")
    w[1] = float("inf")
    y = moe_grouped_matmul(x.to(DEV), w.to(DEV), off.to(DEV))
    dx = moe_grouped_matmul(dy.to(DEV), w.to(DEV), off.to(DEV), w_transposed=True)
    dw = moe_grouped_matmul_dw(x.to(DEV), dy.to(DEV), off.to(DEV))
    keep = torch.tensor(list(range(4, 25)) + list(range(75, 88)))
    small = offsets_of([21, 13])
    for got, (ref, mag), terms in ((y, grouped_reference(x[keep], w[[0, 2]], small), k), (dx, grouped_reference(dy[keep], w[[0, 2]], small, True), n)):
        assert_within(got[keep.to(DEV)], ref, product_error(mag, terms), "rows")
        assert (got[:4] == 0).all() and (got[-6:] == 0).all() and torch.isnan(got[25:75]).all()
    ref, mag = grouped_dw_reference(x[keep], dy[keep], small)
    assert_within(dw[[0, 2]], ref, product_error(mag, 21), "dw")
    assert torch.isnan(dw[1]).all()


@pytest.mark.parametrize("table", [[0, 30, 20, 50, 64], [-5, 10, 90, 40, 64], [64, 0, 64, 0, 64], [100, 200, 300, 400, 500], [-9, -8, -7, -6, -5]])
def test_tables_out_of_order_stay_in_bounds(table):
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    off = torch.tensor(table, dtype=torch.int32)
    x, w, dy = make((64, 72), torch.bfloat16, 12), make((4, 72, 40), torch.bfloat16, 13), make((64, 40), torch.bfloat16, 14)
    y = moe_grouped_matmul(x.to(DEV), w.to(DEV), off.to(DEV))
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, 72), "y")
    dw = moe_grouped_matmul_dw(x.to(DEV), dy.to(DEV), off.to(DEV))
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dw, ref, product_error(mag, 64), "dw")


def test_no_rows():
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    x, w = torch.empty(0, 32, device=DEV), torch.ones(2, 32, 24, device=DEV)
    assert moe_grouped_matmul(x, w, off).shape == (0, 24)
    dw = moe_grouped_matmul_dw(x, torch.empty(0, 24, device=DEV), off, out=torch.full((2, 32, 24), 3.0, device=DEV))
    assert (dw == 0).all()


def test_gradient_against_differences():
    """d/dt of sum(y * dy) along a direction of x and of w, by differences of the plain product in 64 bits."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts = [7, 0, 20]
    off = offsets_of(counts)
    x, w, dy = (make(s, torch.float32, 15 + i) for i, s in enumerate([(27, 33), (3, 33, 29), (27, 29)]))
    vx, vw = (make(t.shape, torch.float32, 30 + i).double() for i, t in enumerate((x, w)))
    dx = moe_grouped_matmul(dy.to(DEV), w.to(DEV), off.to(DEV), w_transposed=True).cpu().double()
    dw = moe_grouped_matmul_dw(x.to(DEV), dy.to(DEV), off.to(DEV)).cpu().double()
    h = 1e-4

    def f(t):
        return (grouped_reference(x.double() + t * vx, w.double() + t * vw, off)[0] * dy.double()).sum()

    slope = float(f(h) - f(-h)) / (2 * h)  # f is of the second degree: the difference is exact up to rounding in 64 bits
    mine = float((dx * vx).sum() + (dw * vw).sum())
    most = float((dx.abs() * vx.abs()).sum() + (dw.abs() * vw.abs()).sum())
    assert abs(mine - slope) <= 2 * (33 + 2) * 2.0 ** -24 * most * 4


def test_other_stream_and_graph():
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts, k, n = [130, 0, 77], 128, 256
    off = offsets_of(counts).to(DEV)
    x, w, dy = (make(s, torch.bfloat16, 40 + i).to(DEV) for i, s in enumerate([(207, k), (3, k, n), (207, n)]))
    want = (moe_grouped_matmul(x, w, off), moe_grouped_matmul(dy, w, off, w_transposed=True), moe_grouped_matmul_dw(x, dy, off))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = moe_grouped_matmul(x, w, off, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])
    graph = torch.cuda.CUDAGraph()
    sx, sdy = torch.zeros_like(x), torch.zeros_like(dy)
    with torch.cuda.graph(graph):
        got = (moe_grouped_matmul(sx, w, off), moe_grouped_matmul(sdy, w, off, w_transposed=True), moe_grouped_matmul_dw(sx, sdy, off))
    for i in range(3):
        sx.copy_(x if i != 1 else -x)
        sdy.copy_(dy)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0] if i != 1 else -want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(got[2], want[2] if i != 1 else -want[2])
        assert torch.equal(moe_grouped_matmul(x, w, off), want[0])


def test_rows_beyond_four_gigabytes():
    """Values of x and y that lie more than 2^32 bytes behind the first."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    R, k, n = 600, 64, 64
    stride = 1 << 22  # 600 rows of 8 MiB
    big = torch.empty(R * stride, dtype=torch.bfloat16, device=DEV)
    xs = big.view(R, stride)
    x, w = make((R, k), torch.bfloat16, 50), make((2, k, n), torch.bfloat16, 51)
    xs[:, :k] = x.to(DEV)
    off = offsets_of([500, 100])
    y = moe_grouped_matmul(xs[:, :k], w.to(DEV), off.to(DEV), out=xs[:, 1024:1024 + n])
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, k), "y")
    dw = moe_grouped_matmul_dw(xs[:, :k], xs[:, :k], off.to(DEV))
    ref, mag = grouped_dw_reference(x, x, off)
    assert_within(dw, ref, product_error(mag, 500), "dw")
    del big, xs
    torch.cuda.empty_cache()


def test_more_columns_than_workgroups_for_each_piece_hold():
    """fp32, 64 groups of a row each, 2^23 outputs a row, one weight for all groups: all of them are written, the last ones too."""
    from paper_2508_18376_amd import moe_grouped_matmul
    G, K, N = 64, 4, 1 << 23
    gen = torch.Generator(device=DEV).manual_seed(60)
    x, w = torch.randn(G, K, generator=gen, device=DEV), torch.randn(1, N, K, generator=gen, device=DEV)
    out = torch.full((G, N), float("nan"), device=DEV)
    moe_grouped_matmul(x, w.expand(G, N, K), torch.arange(G + 1, dtype=torch.int32, device=DEV), w_transposed=True, out=out)
    torch.cuda.synchronize()
    step = 1 << 20
    for c in range(0, N, step):
        wc = w[0, c:c + step].double().t().contiguous()
        ref, mag = x.double() @ wc, x.double().abs() @ wc.abs()
        err = product_error(mag, K)
        assert bool(((out[:, c:c + step].double() - ref).abs() <= err + 2.0 ** -24 * (ref.abs() + err)).all()), c


def test_inside_an_autograd_function():
    """Tensors that need gradients are refused where they are recorded, and the forward and backward of a torch.autograd.Function may call the operators."""
    from paper_2508_18376_amd import DsmoeError, moe_grouped_matmul, moe_grouped_matmul_dw

    class Product(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, offsets):
            ctx.save_for_backward(x, w, offsets)
            return moe_grouped_matmul(x, w, offsets)

        @staticmethod
        def backward(ctx, dy):
            x, w, offsets = ctx.saved_tensors
            return moe_grouped_matmul(dy, w, offsets, w_transposed=True), moe_grouped_matmul_dw(x, dy, offsets), None

    counts = [9, 0, 30]
    off = offsets_of(counts)
    x, w, dy = (make(s, torch.float32, 70 + i) for i, s in enumerate([(39, 24), (3, 24, 40), (39, 40)]))
    xd, wd = x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_()
    with pytest.raises(DsmoeError, match="needs gradients"):
        moe_grouped_matmul(xd, wd, off.to(DEV))
    y = Product.apply(xd, wd, off.to(DEV))
    y.backward(dy.to(DEV))
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, 24), "y")
    ref, mag = grouped_reference(dy, w, off, transposed=True)
    assert_within(xd.grad, ref, product_error(mag, 40), "dx")
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(wd.grad, ref, product_error(mag, 30), "dw")


def test_values_that_a_graph_kept_are_not_overwritten_in_silence():
    """A buffer that a recorded product needs for its gradient, then written as `out`: the backward pass refuses, as after torch's own writes."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw, moe_int8_matmul
    off = offsets_of([4, 2]).to(DEV)
    x, w, dy = torch.ones(6, 16, device=DEV), torch.ones(2, 16, 24, device=DEV), torch.ones(6, 24, device=DEV)
    w8, ws = torch.ones(2, 24, 16, dtype=torch.int8, device=DEV), torch.ones(2, 24, device=DEV)
    for shape, call in (((6, 24), lambda out: moe_grouped_matmul(x, w, off, out=out)), ((2, 16, 24), lambda out: moe_grouped_matmul_dw(x, dy, off, out=out)),
                        ((6, 24), lambda out: moe_int8_matmul(x, w8, ws, off, out=out))):
        leaf, out = torch.ones(shape, device=DEV, requires_grad=True), torch.zeros(shape, device=DEV)
        loss = (leaf * out).sum()
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        with torch.inference_mode():
            kept = torch.zeros(shape, device=DEV)
            call(kept)
        call(kept)
        assert torch.equal(kept, out)


# More pieces of work than workgroups (256), so that each takes several: counts, k, n.
SEVERAL = {
    "tiles_of_256": ([1300, 0, 900, 800], 136, 6000),  # 288 and more (y; dx has few)
    "tiles_of_128": ([65 + i % 3 for i in range(40)], 264, 1800),  # 320; dW 640
    "tiles_of_64_one_stage": ([13 + i * 7 % 52 for i in range(40)], 56, 2056),  # 360
    "tiles_of_64_two_stages": ([13 + i * 7 % 52 for i in range(40)], 72, 2056),
    "tiles_of_64_three_stages": ([13 + i * 7 % 52 for i in range(40)], 192, 2056),
    "tiles_of_64_six_stages": ([13 + i * 7 % 52 for i in range(40)], 328, 2056),
    "tiles_of_64_split": ([13 + i * 7 % 52 for i in range(33)], 1608, 2056),  # 297: the last 41 are cut along the contraction
    "tiles_of_64_dx": ([13 + i * 7 % 52 for i in range(40)], 2056, 328),
    "weights": ([100 + i for i in range(20)], 520, 1288),  # dW: 360, of 2 and 3 stages
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", SEVERAL)
def test_workgroups_that_take_several_tiles(name, dtype):
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts, k, n = SEVERAL[name]
    G, R, off, dt = len(counts), sum(counts) + 9, offsets_of(counts, 2), DTYPES[dtype]
    x, w, dy = make((R, k), dt, 80), make((G, k, n), dt, 81, 0.1), make((R, n), dt, 82)
    xd, wd, dyd, offd = x.to(DEV), w.to(DEV), dy.to(DEV), off.to(DEV)
    print(name, dtype, R, G, k, n, flush=True)
    y, dx, dw = (moe_grouped_matmul(xd, wd, offd), moe_grouped_matmul(dyd, wd, offd, w_transposed=True), moe_grouped_matmul_dw(xd, dyd, offd))
    torch.cuda.synchronize()
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, k), "y")
    ref, mag = grouped_reference(dy, w, off, transposed=True)
    assert_within(dx, ref, product_error(mag, n), "dx")
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dw, ref, product_error(mag, max(counts)), "dw")
    for t in (y, dx):
        assert (t[:2] == 0).all() and (t[2 + sum(counts):] == 0).all()
    for _ in range(3):
        assert torch.equal(y, moe_grouped_matmul(xd, wd, offd)) and torch.equal(dx, moe_grouped_matmul(dyd, wd, offd, w_transposed=True))
        assert torch.equal(dw, moe_grouped_matmul_dw(xd, dyd, offd))


# More groups than a wavefront has lanes, on every kind of tile: counts, k, n.
MANY = {
    "tiles_of_64": ([(13 + i * 7 % 52) * (i % 11 != 3) + 2 for i in range(150)], 72, 264),
    "tiles_of_64_full_groups": ([13 + i * 5 % 40 for i in range(512)], 40, 264),
    "tiles_of_64_split": ([13 + i * 7 % 52 for i in range(65)], 1536, 136),  # y in 3 parts
    "tiles_of_128": ([65 + i % 5 for i in range(150)], 136, 264),
    "tiles_of_128_ragged": ([(i * 37 % 301) * (i % 7 != 2) + 60 for i in range(65)], 72, 264),
    "tiles_of_256": ([65 + i % 9 for i in range(520)], 72, 264),
    "weights_split": ([1000 + i % 50 for i in range(260)], 24, 40),  # dW of the last four in parts
    "odd": ([17 + i % 30 for i in range(150)], 45, 77),
    "odd_few": ([i % 3 for i in range(512)], 45, 77),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", MANY)
def test_more_groups_than_lanes(name, dtype):
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    counts, k, n = MANY[name]
    G, R, off, dt = len(counts), sum(counts) + 9, offsets_of(counts, 2), DTYPES[dtype]
    x, w, dy = make((R, k), dt, 90), make((G, k, n), dt, 91, 0.1), make((R, n), dt, 92)
    xd, wd, dyd, offd = x.to(DEV), w.to(DEV), dy.to(DEV), off.to(DEV)
    print(name, dtype, R, G, k, n, flush=True)
    y, dx, dw = (moe_grouped_matmul(xd, wd, offd), moe_grouped_matmul(dyd, wd, offd, w_transposed=True), moe_grouped_matmul_dw(xd, dyd, offd))
    torch.cuda.synchronize()
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, k), "y")
    ref, mag = grouped_reference(dy, w, off, transposed=True)
    assert_within(dx, ref, product_error(mag, n), "dx")
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dw, ref, product_error(mag, max(counts)), "dw")
    for t in (y, dx):
        assert (t[:2] == 0).all() and (t[2 + sum(counts):] == 0).all()


@pytest.mark.parametrize("k,n", [(72, 40), (45, 77)])
@pytest.mark.parametrize("rows", [400, 6000, 12000])
def test_long_tables_out_of_order_stay_in_bounds(rows, k, n):
    """150 groups whose bounds are any numbers around the rows."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    gen = torch.Generator().manual_seed(rows)
    off = (torch.linspace(-0.1, 1.1, 151) * rows + torch.randn(151, generator=gen) * rows / 40).to(torch.int32)
    x, w, dy = make((rows, k), torch.bfloat16, 93), make((150, k, n), torch.bfloat16, 94), make((rows, n), torch.bfloat16, 95)
    y = moe_grouped_matmul(x.to(DEV), w.to(DEV), off.to(DEV))
    ref, mag = grouped_reference(x, w, off)
    assert_within(y, ref, product_error(mag, k), "y")
    dw = moe_grouped_matmul_dw(x.to(DEV), dy.to(DEV), off.to(DEV))
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dw, ref, product_error(mag, rows), "dw")


def test_tiles_of_rows_beyond_four_gigabytes():
    """Rows exactly 4 MiB apart, the most that the tiles take, and more than 2^32 bytes of them: x, dy, outputs, and the weights' rows too."""
    from paper_2508_18376_amd import moe_grouped_matmul, moe_grouped_matmul_dw
    R, k, n, apart = 1100, 264, 328, 1 << 21
    big = torch.empty(R * apart, dtype=torch.bfloat16, device=DEV).view(R, apart)
    weights = torch.empty(2 * k * apart, dtype=torch.bfloat16, device=DEV).view(2, k, apart)
    x, w, dy = make((R, k), torch.bfloat16, 52), make((2, k, n), torch.bfloat16, 53, 0.1), make((R, n), torch.bfloat16, 54)
    xd, dyd, yd, dxd = (big[:, c:c + v] for c, v in ((0, k), (1024, n), (2048, n), (4096, k)))
    xd.copy_(x)
    dyd.copy_(dy)
    wd, dwd = weights[:, :, :n], weights[:, :, 1024:1024 + n]
    wd.copy_(w)
    off = offsets_of([1000, 100])
    moe_grouped_matmul(xd, wd, off.to(DEV), out=yd)
    moe_grouped_matmul(dyd, wd, off.to(DEV), w_transposed=True, out=dxd)
    moe_grouped_matmul_dw(xd, dyd, off.to(DEV), out=dwd)
    torch.cuda.synchronize()
    ref, mag = grouped_reference(x, w, off)
    assert_within(yd, ref, product_error(mag, k), "y")
    ref, mag = grouped_reference(dy, w, off, transposed=True)
    assert_within(dxd, ref, product_error(mag, n), "dx")
    ref, mag = grouped_dw_reference(x, dy, off)
    assert_within(dwd, ref, product_error(mag, 1000), "dw")
    # tiles of 64 rows: many groups of few rows, all weights the first group's
    counts = [50 + i % 2 for i in range(20)]
    off = offsets_of(counts)
    moe_grouped_matmul(xd, wd[:1].expand(20, k, n), off.to(DEV), out=yd)
    torch.cuda.synchronize()
    ref, mag = grouped_reference(x, w[:1].expand(20, k, n), off)
    assert_within(yd, ref, product_error(mag, k), "y")
    del big, weights, xd, dyd, yd, dxd, wd, dwd
    torch.cuda.empty_cache()
