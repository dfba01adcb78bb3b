"""CPU: calls of the operators beside the layer that do not fit their tensors are refused before anything is launched, in the Python binding and at
the C boundary."""
import ctypes

import pytest
import torch

import paper_2508_18376_amd as ds
from paper_2508_18376_amd import operators as ops
from paper_2508_18376_amd.binding import _lib

I32, BF = torch.int32, torch.bfloat16


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def off(n):
    return torch.zeros(n, dtype=I32)


GROUPED = {
    "x of 3 dimensions": lambda: ds.moe_grouped_matmul(z(1, 4, 8), z(2, 8, 6), off(3)),
    "w of 2 dimensions": lambda: ds.moe_grouped_matmul(z(4, 8), z(8, 6), off(3)),
    "widths differ": lambda: ds.moe_grouped_matmul(z(4, 7), z(2, 8, 6), off(3)),
    "widths differ, transposed": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(3), w_transposed=True),
    "types differ": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6, dtype=torch.float16), off(3)),
    "integers": lambda: ds.moe_grouped_matmul(z(4, 8, dtype=torch.int8), z(2, 8, 6, dtype=torch.int8), off(3)),
    "64-bit values": lambda: ds.moe_grouped_matmul(z(4, 8, dtype=torch.float64), z(2, 8, 6, dtype=torch.float64), off(3)),
    "64-bit offsets": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(3).long()),
    "offsets too short": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(2)),
    "offsets too long": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(4)),
    "offsets with gaps": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(6)[::2]),
    "x by columns": lambda: ds.moe_grouped_matmul(z(8, 4).t(), z(2, 8, 6), off(3)),
    "w by columns": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 6, 8).transpose(1, 2), off(3)),
    "not on a GPU": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 6), off(3)),
    "dw: rows differ": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(5, 6), off(3)),
    "dw: types differ": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(4, 6, dtype=torch.float16), off(3)),
    "dw: one offset": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(4, 6), off(1)),
    "dw: dy by columns": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(6, 4).t(), off(3)),
    "dw: not on a GPU": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(4, 6), off(3)),
    "int8: w in bf16": lambda: ds.moe_int8_matmul(z(4, 8), z(1, 6, 8), z(1, 6, dtype=torch.float32)),
    "int8: x in int8": lambda: ds.moe_int8_matmul(z(4, 8, dtype=torch.int8), z(1, 6, 8, dtype=torch.int8), z(1, 6, dtype=torch.float32)),
    "int8: widths differ": lambda: ds.moe_int8_matmul(z(4, 9), z(1, 6, 8, dtype=torch.int8), z(1, 6, dtype=torch.float32)),
    "int8: scales for too few channels": lambda: ds.moe_int8_matmul(z(4, 8), z(1, 6, 8, dtype=torch.int8), z(1, 5, dtype=torch.float32)),
    "int8: scales in bf16": lambda: ds.moe_int8_matmul(z(4, 8), z(1, 6, 8, dtype=torch.int8), z(1, 6)),
    "int8: groups without offsets": lambda: ds.moe_int8_matmul(z(4, 8), z(2, 6, 8, dtype=torch.int8), z(2, 6, dtype=torch.float32)),
    "int8: not on a GPU": lambda: ds.moe_int8_matmul(z(4, 8), z(1, 6, 8, dtype=torch.int8), z(1, 6, dtype=torch.float32)),
}


def norm(**kw):
    a = dict(x=z(4, 8), branch=z(4, 8), branch_weight=z(8), weight=z(8), gate=None, eps=1e-6)
    a.update(kw)
    return ds.moe_block_norm(a.pop("x"), **a)


NORM = {
    "branch of another shape": dict(branch=z(4, 9)),
    "branch of another type": dict(branch=z(4, 8, dtype=torch.float32)),
    "x of 1 dimension": dict(x=z(8), branch=z(8)),
    "rows without values": dict(x=z(4, 0), branch=z(4, 0), branch_weight=z(0), weight=z(0)),
    "short weight": dict(weight=z(7)),
    "branch_weight by rows": dict(branch_weight=z(1, 8)),
    "gate of 1 dimension": dict(gate=z(8)),
    "gate of one value": dict(gate=z(1, 1)),
    "gate for too few tokens": dict(gate=z(3, 1)),
    "gate of another type": dict(gate=z(4, 1, dtype=torch.float32)),
    "gate by columns": dict(gate=z(8, 4).t()),
    "weights with gaps": dict(weight=z(16)[::2]),
    "negative eps": dict(eps=-1e-6),
    "integers": dict(x=z(4, 8, dtype=I32), branch=z(4, 8, dtype=I32), branch_weight=z(8, dtype=I32), weight=z(8, dtype=I32)),
    "not on a GPU": dict(),
}


@pytest.mark.parametrize("case", GROUPED)
def test_products_refuse(case):
    with pytest.raises(ds.DsmoeError) as e:
        GROUPED[case]()
    assert e.value.status == -1 and "moe_" in str(e.value)


@pytest.mark.parametrize("case", NORM)
def test_norms_refuse(case):
    with pytest.raises(ds.DsmoeError) as e:
        norm(**NORM[case])
    assert e.value.status == -1 and "moe_block_norm" in str(e.value)


@pytest.mark.parametrize("bad", ["dy", "dh", "stats", "stats_type", "type"])
def test_norms_backward_refuses(bad):
    dy, dh, x, stats = z(4, 8), z(4, 8), z(4, 8), z(2, 4, dtype=torch.float32)
    if bad == "dy":
        dy = z(4, 7)
    if bad == "dh":
        dh = z(5, 8)
    if bad == "stats":
        stats = z(4, 2, dtype=torch.float32)
    if bad == "stats_type":
        stats = z(2, 4)
    if bad == "type":
        dy = z(4, 8, dtype=torch.float32)
    with pytest.raises(ds.DsmoeError) as e:
        ds.moe_block_norm_backward(dy, dh, x, stats, branch=z(4, 8), branch_weight=z(8), weight=z(8))
    assert e.value.status == -1


P = 1 << 20  # an address that nothing reads: every call below is refused


def grouped(x=P, xs=64, w=P, wg=64 * 32, wr=32, o=P, rows=10, groups=2, k=64, n=32, t=0, dt=1, y=P, ys=32, work=None):
    return _lib.moe_grouped_matmul(x, xs, w, wg, wr, o, rows, groups, k, n, t, dt, y, ys, work, None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(w=None), dict(o=None), dict(y=None), dict(rows=-1), dict(groups=0), dict(k=0), dict(n=0), dict(t=2),
                                dict(dt=3), dict(dt=-1), dict(xs=-1), dict(wg=-1), dict(wr=-1), dict(ys=31), dict(t=1), dict(x=P + 1), dict(y=P + 1),
                                dict(dt=0, w=P + 2), dict(rows=(1 << 23) + 1), dict(groups=1 << 17), dict(k=(1 << 24) + 1),
                                dict(rows=1 << 23, n=1 << 24, ys=1 << 24), dict(work=P + 128)], ids=str)
def test_grouped_boundary(kw):
    assert grouped(**kw) == -1


def dw(x=P, xs=64, dy=P, ds_=32, o=P, rows=10, groups=2, k=64, n=32, dt=1, out=P, og=64 * 32, orow=32, work=None):
    return _lib.moe_grouped_matmul_dw(x, xs, dy, ds_, o, rows, groups, k, n, dt, out, og, orow, work, None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(dy=None), dict(o=None), dict(out=None), dict(rows=-1), dict(groups=0), dict(k=0), dict(n=0), dict(dt=3),
                                dict(xs=-1), dict(ds_=-1), dict(orow=31), dict(og=64 * 32 - 1), dict(x=P + 1), dict(out=P + 1),
                                dict(k=1 << 24, n=1 << 24, orow=1 << 24, og=1 << 39), dict(work=P + 128)], ids=str)
def test_dw_boundary(kw):
    assert dw(**kw) == -1


def int8(x=P, xs=64, w=P, wg=64 * 32, wr=64, ws=P, wsg=32, o=P, rows=10, groups=2, k=64, n=32, dt=1, y=P, ys=32, work=P):
    return _lib.moe_int8_matmul(x, xs, w, wg, wr, ws, wsg, o, rows, groups, k, n, dt, y, ys, work, None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(w=None), dict(ws=None), dict(y=None), dict(work=None), dict(o=None), dict(rows=-1), dict(groups=0),
                                dict(k=0), dict(k=(1 << 17) + 1), dict(n=0), dict(dt=3), dict(xs=-1), dict(wr=-1), dict(wsg=-1), dict(ys=31),
                                dict(work=P + 128), dict(ws=P + 2), dict(x=P + 1)], ids=str)
def test_int8_boundary(kw):
    assert int8(**kw) == -1


def test_workspace_sizes():
    assert _lib.dsmoe_int8_workspace_bytes(10, 1, 64, 32) >= 10 * 64 + 40
    assert _lib.dsmoe_int8_workspace_bytes(-1, 1, 64, 32) == 0 and _lib.dsmoe_int8_workspace_bytes(10, 1, 0, 32) == 0
    # few rows, and sums too short to be worth it, are not split; few tiles of long sums are
    assert _lib.dsmoe_grouped_workspace_bytes(8, 64, 2048, 1024, 0, 1) == 0 and _lib.dsmoe_grouped_workspace_bytes(4096, 8, 256, 1024, 0, 1) == 0
    assert _lib.dsmoe_grouped_workspace_bytes(512, 1, 14336, 512, 0, 1) > 0 and _lib.dsmoe_grouped_workspace_bytes(512, 1, 14336, 512, 0, 0) == 0
    assert _lib.dsmoe_grouped_dw_workspace_bytes(65536, 1, 256, 256, 1) > 0 and _lib.dsmoe_grouped_dw_workspace_bytes(128, 8, 256, 256, 1) == 0
    a = ops._BlockNormArgs(100, 64, 1, 2, 1.0, 0.0, 1e-6, 0, 64, 64, 0, 64, 64)
    assert _lib.dsmoe_block_norm_workspace_bytes(a) >= 3 * 64 * 4
    a.gate_kind = 4
    assert _lib.dsmoe_block_norm_workspace_bytes(a) == 0 and _lib.dsmoe_block_norm_workspace_bytes(None) == 0


NORM_ARGS = dict(tokens=4, d=8, dtype=1, gate_kind=0, scale=1.0, weight_offset=0.0, eps=1e-6, pad=0, x_stride=8, branch_stride=8, gate_stride=0, dy_stride=8,
                 dh_stride=8)


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(d=0), dict(dtype=3), dict(gate_kind=-1), dict(gate_kind=4), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(x_stride=-1), dict(branch_stride=-1), dict(gate_stride=-1), dict(gate_kind=1)], ids=str)
def test_norm_boundary(kw):
    a = ops._BlockNormArgs(**dict(NORM_ARGS, **kw))
    assert _lib.moe_block_norm(a, P, P, P, None, P, P, P, P, None) == -1
    assert _lib.moe_block_norm_backward(a, P, P, P, P, P, None, P, P, P, P, P, None, P, P, None) == -1


def test_norm_pointers():
    a = ops._BlockNormArgs(**NORM_ARGS)
    good = [P, P, P, None, P, P, P]
    for i in (0, 1, 2, 4, 5, 6):
        for bad in (None, P + 1):
            p = list(good)
            p[i] = bad
            assert _lib.moe_block_norm(a, *p, P, None) == -1
    assert _lib.moe_block_norm(a, P, P, P, P, P, P, P, P, None) == -1  # a gate where there is none
    assert _lib.moe_block_norm(None, *good, P, None) == -1
    good = [P, P, P, P, P, None, P, P, P, P, P, None, P, P]
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9, 10, 12, 13):
        p = list(good)
        p[i] = None
        assert _lib.moe_block_norm_backward(a, *p, None) == -1
    p = list(good)
    p[13] = P + 64
    assert _lib.moe_block_norm_backward(a, *p, None) == -1


def test_errors_without_a_context_are_kept():
    _lib.dsmoe_last_hip_error.restype = ctypes.c_int
    assert _lib.dsmoe_last_hip_error(None) == 0


def test_calls_too_large_for_a_workgroup_for_each_piece_go_to_the_tiles():
    """A launch of 2^32 threads is cut short, and the kernels for groups of few rows have 512 threads (across: 256) for 64 (128) columns of 32 rows.
    Which kernels a call goes to shows in the workspace: they split nothing, the tiles do."""
    def int8_split(rows, groups, k, n):
        held = (rows * ((k + 127) // 128 * 128) + 255) // 256 * 256 + (rows * 4 + 255) // 256 * 256
        return _lib.dsmoe_int8_workspace_bytes(rows, groups, k, n) - held

    k = 2048
    assert int8_split(64, 64, k, (1 << 23) - 64) == 0 and int8_split(64, 64, k, 1 << 23) > 0
    assert int8_split(1 << 16, 1 << 16, k, 8192 - 64) == 0 and int8_split(1 << 16, 1 << 16, k, 8192) > 0
    assert int8_split(64, 64, k, 1 << 24) > 0
    bf16 = _lib.dsmoe_grouped_workspace_bytes
    assert bf16(64, 64, 1 << 22, k, 1, 1) == 0 and bf16(64, 64, 1 << 23, k, 1, 1) > 0  # along
    assert bf16(64, 64, k, 1 << 23, 0, 1) == 0  # across: half as many pieces, of half as many threads


MANY = (1 << 32) + 5  # 5, if cut off to 32 bits
SIZES = {
    "rows": lambda: ds.moe_grouped_matmul(z(1, 8).expand(MANY, 8), z(2, 8, 6), off(3)),
    "columns": lambda: ds.moe_grouped_matmul(z(4, 8), z(2, 8, 1).expand(2, 8, MANY), off(3)),
    "dw: rows": lambda: ds.moe_grouped_matmul_dw(z(1, 8).expand(MANY, 8), z(1, 6).expand(MANY, 6), off(3)),
    "dw: columns": lambda: ds.moe_grouped_matmul_dw(z(4, 8), z(4, 1).expand(4, MANY), off(3)),
    "int8: rows": lambda: ds.moe_int8_matmul(z(1, 8).expand(MANY, 8), z(1, 6, 8, dtype=torch.int8), z(1, 6, dtype=torch.float32)),
    "int8: columns": lambda: ds.moe_int8_matmul(z(4, 8), z(1, 1, 8, dtype=torch.int8).expand(1, MANY, 8), z(1, 1, dtype=torch.float32).expand(1, MANY)),
    "norm: tokens": lambda: norm(x=z(1, 8).expand(MANY, 8), branch=z(1, 8).expand(MANY, 8)),
    "norm: width": lambda: norm(x=z(1, 1).expand(1, MANY), branch=z(1, 1).expand(1, MANY), branch_weight=z(1).expand(MANY), weight=z(1).expand(MANY)),
}


@pytest.mark.parametrize("case", SIZES)
def test_sizes_beyond_32_bits_are_refused(case):
    with pytest.raises(ds.DsmoeError, match="2\\^31") as e:
        SIZES[case]()
    assert e.value.status == -1


def _calls():
    """Each operator with its tensors by name, and which of them a gradient can go to."""
    f32 = torch.float32
    nm = dict(x=z(4, 8), branch=z(4, 8), branch_weight=z(8), weight=z(8), gate=z(4, 1))
    return {
        "moe_grouped_matmul": (lambda a: ds.moe_grouped_matmul(a["x"], a["w"], off(3), out=a["out"]), dict(x=z(4, 8), w=z(2, 8, 6), out=z(4, 6))),
        "moe_grouped_matmul_dw": (lambda a: ds.moe_grouped_matmul_dw(a["x"], a["dy"], off(3), out=a["out"]), dict(x=z(4, 8), dy=z(4, 6), out=z(2, 8, 6))),
        "moe_int8_matmul": (lambda a: ds.moe_int8_matmul(a["x"], z(1, 6, 8, dtype=torch.int8), a["w_scale"], out=a["out"]),
                            dict(x=z(4, 8), w_scale=z(1, 6, dtype=f32), out=z(4, 6))),
        "moe_block_norm": (lambda a: ds.moe_block_norm(a.pop("x"), **a), nm),
        "moe_block_norm_backward": (lambda a: ds.moe_block_norm_backward(*[a.pop(n) for n in ("dy", "dh", "x", "stats")], **a),
                                    dict(nm, dy=z(4, 8), dh=z(4, 8), stats=z(2, 4, dtype=f32))),
    }


@pytest.mark.parametrize("op,name", [(op, name) for op, (_, tensors) in _calls().items() for name in tensors])
def test_nothing_is_cut_from_the_graph_in_silence(op, name):
    """A tensor that needs gradients, or has a tangent, is refused while they are recorded.  (Where they are not, the next check refuses: no GPU here.)"""
    def refusal(change):
        call, tensors = _calls()[op]
        tensors[name] = change(tensors[name])
        with pytest.raises(ds.DsmoeError) as e:
            call(tensors)
        assert e.value.status == -1 and op in str(e.value)
        return str(e.value)

    assert "needs gradients" in refusal(lambda t: t.requires_grad_())
    assert "needs gradients" in refusal(lambda t: t.requires_grad_() * 1)  # not a leaf
    with torch.no_grad():
        assert "on one GPU" in refusal(lambda t: t.requires_grad_())
    assert "on one GPU" in refusal(lambda t: t)
    with torch.autograd.forward_ad.dual_level():
        assert "tangent" in refusal(lambda t: torch.autograd.forward_ad.make_dual(t, torch.ones_like(t)))
        assert "on one GPU" in refusal(lambda t: t)


class OnGpu0:
    """A CPU tensor that says it lies on the first GPU: the checks up to the stream's read nothing of it."""
    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


class Stream1:
    device = torch.device("cuda", 1)


@pytest.mark.parametrize("op", ["moe_grouped_matmul", "moe_grouped_matmul_dw", "moe_int8_matmul", "moe_block_norm", "moe_block_norm_backward"])
def test_streams_of_another_gpu_are_refused(op, monkeypatch):
    """The call would run on the tensors' GPU, on a stream that the caller did not name."""
    monkeypatch.setattr(ops, "_current_device", lambda: 0)

    def refuse(*_):
        raise AssertionError("the named stream is entered, though it is another GPU's")

    monkeypatch.setattr(torch.cuda, "stream", refuse)
    norms = {k: OnGpu0(v) for k, v in dict(branch=z(4, 8), branch_weight=z(8), weight=z(8)).items()}
    x, o = OnGpu0(z(4, 8)), OnGpu0(off(3))
    with pytest.raises(ds.DsmoeError, match="stream") as e:
        if op == "moe_grouped_matmul":
            ds.moe_grouped_matmul(x, OnGpu0(z(2, 8, 6)), o, stream=Stream1())
        elif op == "moe_grouped_matmul_dw":
            ds.moe_grouped_matmul_dw(x, OnGpu0(z(4, 6)), o, stream=Stream1())
        elif op == "moe_int8_matmul":
            ds.moe_int8_matmul(x, OnGpu0(z(1, 6, 8, dtype=torch.int8)), OnGpu0(z(1, 6, dtype=torch.float32)), stream=Stream1())
        elif op == "moe_block_norm":
            ds.moe_block_norm(x, stream=Stream1(), **norms)
        else:
            ds.moe_block_norm_backward(OnGpu0(z(4, 8)), OnGpu0(z(4, 8)), x, OnGpu0(z(2, 4, dtype=torch.float32)), stream=Stream1(), **norms)
    assert e.value.status == -1 and op in str(e.value)
