"""The gated half of a block and its gradients against plain formulas in 64 bits: types, activations, odd and aligned sizes, ragged, empty and missing groups,
strides, streams, graphs, tables out of order."""
import pytest
import torch

from gated_util import activation, reference
from operator_util import DTYPES, assert_within, offsets_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(shape, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * std).to(dtype)


def tensors(R, G, k, n, dt, seed=1):
    """x, w1, w3, dh: weights so that the products are of order one, in all of the activation's curve."""
    return make((R, k), dt, seed), make((G, k, n), dt, seed + 1, 1.5 * k ** -0.5), make((G, k, n), dt, seed + 2, k ** -0.5), make((R, n), dt, seed + 3)


def both(x, w1, w3, off, kind, dh):
    """Forward and backward on the GPU: {"h", "saved", "dx", "dw1", "dw3"}."""
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    h, saved = moe_gated_matmul(x, w1, w3, off, activation=kind, want_saved=True)
    torch.cuda.synchronize()
    out = dict(h=h, saved=saved, **moe_gated_matmul_backward(dh, x, w1, w3, saved, off, activation=kind))
    torch.cuda.synchronize()
    return out


def check(got, want, held):
    """held: the rows that a group has."""
    for name, (ref, err) in want.items():
        if name == "saved":
            assert_within(got[name][:, held], ref[:, held], err[:, held], name)
        else:
            assert_within(got[name], ref, err, name)


def rows_held(R, before, count):
    held = torch.zeros(R, dtype=torch.bool)
    held[before:before + count] = True
    return held


# counts of the groups, rows in front of the first and behind the last one, k, n
SHAPES = {
    "one_row": ([1], 0, 0, 64, 64),
    "one_value": ([1], 0, 0, 1, 1),
    "few_of_many": ([0, 1, 0, 2, 0, 0, 1, 0], 0, 0, 256, 192),
    "decode": ([1, 0, 2, 1, 0, 3, 0, 1], 0, 0, 512, 384),
    "sixteens": ([16, 17, 15, 32, 33], 0, 0, 320, 264),
    "few_many_columns": ([3, 2], 2, 1, 72, 20000),
    "ragged": ([70, 0, 129, 1, 255], 3, 5, 136, 200),
    "spare_ends": ([5, 300], 17, 41, 64, 328),
    "tiles_128": ([256, 512, 64], 0, 0, 256, 512),
    "tiles_256": ([2100, 300, 1900], 0, 3, 136, 1032),
    "narrow": ([300, 100], 0, 0, 72, 40),
    "half_tile_columns": ([300, 100], 0, 0, 72, 192),
    "long_k": ([40, 9], 0, 0, 2048, 96),
    "long_rows": ([1500, 700], 0, 0, 72, 136),
    "odd": ([37, 0, 131, 6], 2, 3, 101, 77),
    "odd_k": ([65, 64], 0, 0, 203, 128),
    "odd_n": ([65, 64], 0, 0, 128, 203),
    "even_not_aligned": ([90, 45], 0, 1, 130, 166),
    "odd_many_rows": ([300, 290], 1, 0, 61, 333),
    "no_rows_in_groups": ([0, 0, 0], 4, 9, 64, 72),
    "split_k": ([300, 0, 40, 70], 5, 9, 4096, 264),
    "split_n": ([300, 0, 40, 70], 5, 9, 264, 4096),
    "split_n_not_in_stages": ([300, 0, 40, 70], 5, 9, 264, 4136),
    "split_short": ([50, 20, 0, 30], 5, 9, 520, 4136),
    "split_rows": ([5000, 0, 1234], 1, 2, 264, 136),
    "split_last_round": ([4200, 3900], 0, 60, 520, 1160),
    "many_groups": ([i % 3 for i in range(150)], 1, 0, 64, 40),
    "many_groups_tiles": ([65 + i % 5 for i in range(150)], 0, 7, 72, 136),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
def test_forward_and_gradients(name, dtype):
    from paper_2508_18376_amd import moe_gated_matmul
    counts, before, after, k, n = SHAPES[name]
    dt, off, kind = DTYPES[dtype], offsets_of(counts, before), "gelu_tanh" if len(name) % 2 else "silu"
    R, G = before + sum(counts) + after, len(counts)
    x, w1, w3, dh = tensors(R, G, k, n, dt)
    xd, ud, vd, dd, od = (t.to(DEV) for t in (x, w1, w3, dh, off))
    print(name, dtype, kind, R, G, k, n, flush=True)
    got = both(xd, ud, vd, od, kind, dd)
    held = rows_held(R, before, sum(counts))
    check(got, reference(x, w1, w3, off, kind, dh), held)
    assert (got["h"].cpu()[~held] == 0).all() and (got["dx"].cpu()[~held] == 0).all()
    # the same inputs give the same bits, with and without what the backward pass takes
    assert torch.equal(got["h"], moe_gated_matmul(xd, ud, vd, od, activation=kind))
    again = both(xd, ud, vd, od, kind, dd)
    assert all(torch.equal(got[name], again[name]) for name in ("h", "dx", "dw1", "dw3"))


# More pieces of work than workgroups (256), so that each takes several: counts, k, n.
SEVERAL = {
    "tiles_of_256": ([1300, 0, 900, 800], 136, 3400),
    "tiles_of_128": ([65 + i % 3 for i in range(40)], 264, 904),
    "tiles_of_64_one_stage": ([13 + i * 7 % 52 for i in range(40)], 56, 1032),
    "tiles_of_64_six_stages": ([13 + i * 7 % 52 for i in range(40)], 328, 1032),
    "tiles_of_64_split": ([13 + i * 7 % 52 for i in range(33)], 1608, 1032),
    "tiles_of_64_dx": ([13 + i * 7 % 52 for i in range(40)], 2056, 168),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", SEVERAL)
def test_workgroups_that_take_several_tiles(name, dtype):
    counts, k, n = SEVERAL[name]
    G, R, off, dt = len(counts), sum(counts) + 9, offsets_of(counts, 2), DTYPES[dtype]
    x, w1, w3, dh = tensors(R, G, k, n, dt, 10)
    print(name, dtype, R, G, k, n, flush=True)
    dev = [t.to(DEV) for t in (x, w1, w3, off, dh)]
    got = both(*dev[:4], "silu", dev[4])
    check(got, reference(x, w1, w3, off, "silu", dh), rows_held(R, 2, sum(counts)))
    for _ in range(2):
        again = both(*dev[:4], "silu", dev[4])
        assert all(torch.equal(got[name], again[name]) for name in ("h", "dx", "dw1", "dw3"))


@pytest.mark.parametrize("rows", [1, 20, 700])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_group_without_a_table(rows, dtype):
    dt = DTYPES[dtype]
    x, w1, w3, dh = tensors(rows, 1, 200, 1096, dt, 20)
    got = both(x.to(DEV), w1.to(DEV), w3.to(DEV), None, "silu", dh.to(DEV))
    check(got, reference(x, w1, w3, None, "silu", dh), rows_held(rows, 0, rows))
    off = offsets_of([rows]).to(DEV)
    again = both(x.to(DEV), w1.to(DEV), w3.to(DEV), off, "silu", dh.to(DEV))
    assert all(torch.equal(got[name], again[name]) for name in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [8, 3])
def test_strided_rows(dtype, pad):
    """Inputs inside wider tensors, both weights side by side in one, an output into a wider tensor, whose other values stay."""
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    dt, k, n = DTYPES[dtype], 96, 160
    counts = [33, 0, 140]
    R, off = sum(counts), offsets_of(counts)
    x, w, dh = make((R, k + pad), dt, 30), make((3, k + 1, 2 * n + pad), dt, 31, 0.1), make((R, n + pad), dt, 32)
    xd, wd, dd, od = (t.to(DEV) for t in (x, w, dh, off))
    wide = torch.full((R, n + pad), 7.0, dtype=dt, device=DEV)
    how = (xd[:, :k], wd[:, :k, :n], wd[:, :k, n:2 * n])
    h, saved = moe_gated_matmul(*how, od, want_saved=True, out=wide[:, :n])
    assert h.data_ptr() == wide.data_ptr() and (wide[:, n:] == 7).all()
    got = dict(h=h, saved=saved, **moe_gated_matmul_backward(dd[:, :n], *how, saved, od))
    check(got, reference(x[:, :k], w[:, :k, :n], w[:, :k, n:2 * n], off, "silu", dh[:, :n]), rows_held(R, 0, R))


def test_rows_and_weights_that_overlap():
    """Strides of zero: one row for all tokens, one weight for all groups, the same for both projections."""
    off = offsets_of([40, 30])
    x, w, dh = make((1, 64), torch.bfloat16, 40), make((1, 64, 72), torch.bfloat16, 41, 0.2), make((1, 72), torch.bfloat16, 42)
    xd, wd, dd = x.to(DEV).expand(70, 64), w.to(DEV).expand(2, 64, 72), dh.to(DEV).expand(70, 72)
    got = both(xd, wd, wd, off.to(DEV), "silu", dd)
    check(got, reference(x.expand(70, 64), w.expand(2, 64, 72), w.expand(2, 64, 72), off, "silu", dh.expand(70, 72)), rows_held(70, 0, 70))


@pytest.mark.parametrize("k", [64, 61])
def test_other_groups_values_do_not_leak(k):
    """NaN and infinities in one group's rows or weights, and in rows of no group, stay out of the other groups' results and gradients."""
    counts, n = [21, 50, 13], 88
    off = offsets_of(counts, 4)
    R = 4 + sum(counts) + 6
    x, w1, w3, dh = tensors(R, 3, k, n, torch.bfloat16, 50)
    for t in (x, dh):
        t[:4], t[-6:], t[25:75] = float("nan"), float("inf"), float("nan")
    w1[1], w3[1] = float("inf"), float("nan")
    got = both(x.to(DEV), w1.to(DEV), w3.to(DEV), off.to(DEV), "silu", dh.to(DEV))
    keep = torch.tensor(list(range(4, 25)) + list(range(75, 88)))
    small = offsets_of([21, 13])
    want = reference(x[keep], w1[[0, 2]], w3[[0, 2]], small, "silu", dh[keep])
    for name in ("h", "dx"):
        t = got[name].cpu()
        assert_within(t[keep], *want[name], name)
        assert (t[:4] == 0).all() and (t[-6:] == 0).all() and torch.isnan(t[25:75]).all()
    for name in ("dw1", "dw3"):
        assert_within(got[name][[0, 2]], *want[name], name)
        assert torch.isnan(got[name][1]).all()


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_far_out(kind, dtype):
    """First products from -1e30 to 1e30: f saturates without a NaN, and so does its slope."""
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    a = torch.tensor([0.0, 1e-30, 1.0, 20.0, 88.0, 89.0, 105.0, 1e4, 1e13, 1e30])
    a = torch.cat([a, -a]).to(DTYPES[dtype])
    x, w1, w3 = torch.ones(3, 1, dtype=a.dtype), a.view(1, 1, -1), torch.full((1, 1, a.numel()), 0.5, dtype=a.dtype)
    dh = torch.ones(3, a.numel(), dtype=a.dtype)
    h, saved = moe_gated_matmul(x.to(DEV), w1.to(DEV), w3.to(DEV), activation=kind, want_saved=True)
    want = reference(x, w1, w3, None, kind, dh)
    assert_within(h, *want["h"], "h")
    g = moe_gated_matmul_backward(dh.to(DEV), x.to(DEV), w1.to(DEV), w3.to(DEV), saved, activation=kind)
    far = a.double().abs() > 1e12  # (there a s (1 - s) z' of the reference is infinity times zero)
    slope = torch.where(far, (a > 0).double(), activation(a.double(), kind)[1])
    got = g["dw1"].cpu().double().flatten()
    assert ((got - 3 * 0.5 * slope).abs() <= 3 * 0.5 * (2.0 ** -7 if dtype == "bf16" else 1e-4) * slope.abs().clamp_min(1e-3)).all()


@pytest.mark.parametrize("table", [[0, 30, 20, 50, 64], [-5, 10, 90, 40, 64], [64, 0, 64, 0, 64], [100, 200, 300, 400, 500], [-9, -8, -7, -6, -5]])
@pytest.mark.parametrize("k", [72, 45])
def test_tables_out_of_order_stay_in_bounds(table, k):
    off = torch.tensor(table, dtype=torch.int32)
    x, w1, w3, dh = tensors(64, 4, k, 40, torch.bfloat16, 60)
    got = both(x.to(DEV), w1.to(DEV), w3.to(DEV), off.to(DEV), "silu", dh.to(DEV))
    want = reference(x, w1, w3, off, "silu", dh)
    for name in ("h", "dx", "dw1", "dw3"):
        assert_within(got[name], *want[name], name)


def test_no_rows():
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    x, w = torch.empty(0, 32, device=DEV), torch.ones(2, 32, 24, device=DEV)
    h, saved = moe_gated_matmul(x, w, w, off, want_saved=True)
    assert h.shape == (0, 24) and saved.shape == (2, 0, 24)
    g = moe_gated_matmul_backward(h, x, w, w, saved, off)
    assert g["dx"].shape == (0, 32) and (g["dw1"] == 0).all() and (g["dw3"] == 0).all()


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh"])
def test_gradient_against_differences(kind):
    """d/dt of sum(h * dh) along a direction of x, w1 and w3, by central differences of the plain formula in 64 bits: their own error is of order t^2 times the
    third derivative, here below 1e-7 of the slope's terms; the operators' is that of fp32 sums of 33 and 58 terms."""
    counts = [7, 0, 20]
    off = offsets_of(counts)
    x, w1, w3, dh = tensors(27, 3, 33, 29, torch.float32, 70)
    got = {k: v.cpu().double() for k, v in both(x.to(DEV), w1.to(DEV), w3.to(DEV), off.to(DEV), kind, dh.to(DEV)).items()}
    vs = [make(t.shape, torch.float32, 80 + i).double() for i, t in enumerate((x, w1, w3))]
    t = 1e-4

    def f(t):
        moved = [p.double() + t * v for p, v in zip((x, w1, w3), vs)]
        return (reference(*moved, off, kind)["h"][0] * dh.double()).sum()

    slope = float(f(t) - f(-t)) / (2 * t)
    pairs = list(zip((got["dx"], got["dw1"], got["dw3"]), vs))
    mine, most = sum(float((g * v).sum()) for g, v in pairs), sum(float((g.abs() * v.abs()).sum()) for g, v in pairs)
    assert abs(mine - slope) <= (2 * 60 * 2.0 ** -24 * 8 + 1e-6) * most


def test_other_stream_and_graph():
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    counts, k, n = [130, 0, 77], 128, 2304
    off = offsets_of(counts).to(DEV)
    x, w1, w3, dh = (t.to(DEV) for t in tensors(207, 3, k, n, torch.bfloat16, 90))
    want, negated = both(x, w1, w3, off, "silu", dh), both(x, w1, w3, off, "silu", -dh)  # (not the same bits negated: the matrix instructions' sums are not)
    side = torch.cuda.Stream()
    h, saved = moe_gated_matmul(x, w1, w3, off, want_saved=True, stream=side)
    g = moe_gated_matmul_backward(dh, x, w1, w3, saved, off, stream=side)
    side.synchronize()
    assert torch.equal(h, want["h"]) and all(torch.equal(g[name], want[name]) for name in g)
    graph = torch.cuda.CUDAGraph()
    sx, sdh = torch.zeros_like(x), torch.zeros_like(dh)
    with torch.cuda.graph(graph):
        h, saved = moe_gated_matmul(sx, w1, w3, off, want_saved=True)
        g = moe_gated_matmul_backward(sdh, sx, w1, w3, saved, off)
    for i in range(3):
        sx.copy_(x)
        sdh.copy_(dh if i != 1 else -dh)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want["h"])
        for name in g:
            assert torch.equal(g[name], (want if i != 1 else negated)[name])
        assert torch.equal(moe_gated_matmul(x, w1, w3, off), want["h"])


def test_rows_beyond_four_gigabytes():
    """Rows exactly 4 MiB apart, the most that the tiles take, and more than 2^32 bytes of them: x, dh, h, and the weights' rows too."""
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    R, k, n, apart = 1100, 264, 328, 1 << 21
    big = torch.empty(R * apart, dtype=torch.bfloat16, device=DEV).view(R, apart)
    weights = torch.empty(2 * k * apart, dtype=torch.bfloat16, device=DEV).view(2, k, apart)
    x, w1, w3, dh = tensors(R, 2, k, n, torch.bfloat16, 100)
    xd, dd, hd = (big[:, c:c + v] for c, v in ((0, k), (1024, n), (2048, n)))
    xd.copy_(x)
    dd.copy_(dh)
    ud, vd = weights[:, :, :n], weights[:, :, 1024:1024 + n]
    ud.copy_(w1)
    vd.copy_(w3)
    off = offsets_of([1000, 100])
    _, saved = moe_gated_matmul(xd, ud, vd, off.to(DEV), want_saved=True, out=hd)
    got = dict(h=hd, saved=saved, **moe_gated_matmul_backward(dd, xd, ud, vd, saved, off.to(DEV)))
    torch.cuda.synchronize()
    check(got, reference(x, w1, w3, off, "silu", dh), rows_held(R, 0, R))
    # rows further apart go to the other paths, which also pass 2^32
    far = big.view(R // 2, 2 * apart)[:, :k]
    far.copy_(x[:R // 2])
    off = offsets_of([400, 150])
    h = moe_gated_matmul(far, ud, vd, off.to(DEV))
    assert_within(h, *reference(x[:R // 2], w1, w3, off, "silu")["h"], "h")
    del big, weights, xd, dd, hd, ud, vd, far, got
    torch.cuda.empty_cache()


def test_inside_an_autograd_function():
    from paper_2508_18376_amd import DsmoeError, moe_gated_matmul, moe_gated_matmul_backward

    class Gated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w1, w3, offsets):
            h, saved = moe_gated_matmul(x, w1, w3, offsets, want_saved=True)
            ctx.save_for_backward(x, w1, w3, saved, offsets)
            return h

        @staticmethod
        def backward(ctx, dh):
            x, w1, w3, saved, offsets = ctx.saved_tensors
            g = moe_gated_matmul_backward(dh, x, w1, w3, saved, offsets)
            return g["dx"], g["dw1"], g["dw3"], None

    off = offsets_of([9, 0, 30])
    x, w1, w3, dh = tensors(39, 3, 24, 40, torch.float32, 110)
    leaves = [t.to(DEV).requires_grad_() for t in (x, w1, w3)]
    with pytest.raises(DsmoeError, match="needs gradients"):
        moe_gated_matmul(*leaves, off.to(DEV))
    h = Gated.apply(*leaves, off.to(DEV))
    h.backward(dh.to(DEV))
    want = reference(x, w1, w3, off, "silu", dh)
    assert_within(h, *want["h"], "h")
    for t, name in zip(leaves, ("dx", "dw1", "dw3")):
        assert_within(t.grad, *want[name], name)


def test_values_that_a_graph_kept_are_not_overwritten_in_silence():
    from paper_2508_18376_amd import moe_gated_matmul
    x, w = torch.ones(6, 16, device=DEV), torch.ones(1, 16, 24, device=DEV)
    leaf, out = torch.ones(6, 24, device=DEV, requires_grad=True), torch.zeros(6, 24, device=DEV)
    loss = (leaf * out).sum()
    moe_gated_matmul(x, w, w, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_second_gradient_that_starts_anywhere():
    """The C call with dw3 two bytes behind 16: the same values as on 16 bytes, within the products' bounds, and nothing around them."""
    from paper_2508_18376_amd import operators as ops
    counts, k, n = [70, 0, 129], 136, 200
    off, R = offsets_of(counts), sum(counts)
    x, w1, w3, dh = tensors(R, 3, k, n, torch.bfloat16, 60)
    xd, ud, vd, dd, od = (t.to(DEV) for t in (x, w1, w3, dh, off))
    _, saved = ops.moe_gated_matmul(xd, ud, vd, od, want_saved=True)
    dx, dw1, wide = torch.empty_like(xd), torch.empty_like(ud), torch.full((3 * k * n + 2,), 7.0, dtype=torch.bfloat16, device=DEV)
    args = ops._GatedArgs(R, 3, k, n, 1, 0, k, k * n, n, n)
    size = ops._lib.dsmoe_gated_backward_workspace_bytes(args)
    workspace = torch.empty(size, dtype=torch.uint8, device=DEV)
    rc = ops._lib.moe_gated_matmul_backward(args, dd.data_ptr(), xd.data_ptr(), ud.data_ptr(), vd.data_ptr(), saved.data_ptr(), od.data_ptr(), dx.data_ptr(),
                                            dw1.data_ptr(), wide.data_ptr() + 2, workspace.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and wide[0] == 7 and wide[-1] == 7
    want = reference(x, w1, w3, off, "silu", dh)
    for name, got in (("dx", dx), ("dw1", dw1), ("dw3", wide[1:-1].view(3, k, n))):
        assert_within(got, *want[name], name)


def test_as_many_tiles_of_gradients_as_there_may_be():
    """2^23 tiles of 128 columns for each weight: 65536 groups of one value by 16384, of which three have rows."""
    G, n, at = 65536, 16384, {0: 2, 40000: 1, 65535: 3}
    ends = torch.zeros(G + 1, dtype=torch.int64)
    for g, rows in at.items():
        ends[g + 1:] += rows
    x, dh = make((6, 1), torch.float16, 61), make((6, n), torch.float16, 62)
    w1, w3 = (torch.zeros(G, 1, n, dtype=torch.float16, device=DEV) for _ in range(2))
    some = {g: (make((1, n), torch.float16, 63 + g), make((1, n), torch.float16, 64 + g)) for g in at}
    for g, (u, v) in some.items():
        w1[g], w3[g] = u.to(DEV), v.to(DEV)
    got = both(x.to(DEV), w1, w3, ends.int().to(DEV), "silu", dh.to(DEV))
    small = torch.stack([u for u, _ in some.values()]), torch.stack([v for _, v in some.values()])
    want = reference(x, *small, offsets_of(list(at.values())), "silu", dh)
    for name in ("h", "dx"):
        assert_within(got[name], *want[name], name)
    for name in ("dw1", "dw3"):
        for i, g in enumerate(at):
            assert_within(got[name][g], want[name][0][i], want[name][1][i], name)
            got[name][g] = 0
        assert not got[name].any(), name
    del got, w1, w3
    torch.cuda.empty_cache()
