"""CPU: calls of the gated products that do not fit their tensors are refused before anything is launched, in the Python binding and at the C boundary."""
import pytest
import torch

import paper_2508_18376_amd as ds
from paper_2508_18376_amd import operators as ops
from paper_2508_18376_amd.binding import _lib

I32, BF, F32 = torch.int32, torch.bfloat16, torch.float32
MANY = (1 << 32) + 5  # 5, if cut off to 32 bits


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def off(n):
    return torch.zeros(n, dtype=I32)


FORWARD = {
    "x of 3 dimensions": dict(x=z(1, 4, 8)),
    "w1 of 2 dimensions": dict(w1=z(8, 6), w3=z(8, 6)),
    "weights of two shapes": dict(w3=z(2, 8, 5)),
    "widths differ": dict(x=z(4, 7)),
    "types differ": dict(w3=z(2, 8, 6, dtype=torch.float16)),
    "integers": dict(x=z(4, 8, dtype=torch.int8), w1=z(2, 8, 6, dtype=torch.int8), w3=z(2, 8, 6, dtype=torch.int8)),
    "64-bit values": dict(x=z(4, 8, dtype=torch.float64), w1=z(2, 8, 6, dtype=torch.float64), w3=z(2, 8, 6, dtype=torch.float64)),
    "64-bit offsets": dict(offsets=off(3).long()),
    "offsets too short": dict(offsets=off(2)),
    "offsets with gaps": dict(offsets=off(6)[::2]),
    "groups without offsets": dict(offsets=None),
    "an unknown activation": dict(activation="relu"),
    "x by columns": dict(x=z(8, 4).t()),
    "w1 by columns": dict(w1=z(2, 6, 8).transpose(1, 2)),
    "w3 by columns": dict(w3=z(2, 6, 8).transpose(1, 2)),
    "weights with rows of two strides": dict(w3=z(2, 8, 7)[:, :, :6]),
    "weights with groups of two strides": dict(w3=z(2, 9, 6)[:, :8]),
    "not on a GPU": dict(),
}
SIZES = {
    "rows": dict(x=z(1, 8).expand(MANY, 8)),
    "columns": dict(w1=z(2, 8, 1).expand(2, 8, MANY), w3=z(2, 8, 1).expand(2, 8, MANY)),
}


def forward(**kw):
    return ds.moe_gated_matmul(**dict(dict(x=z(4, 8), w1=z(2, 8, 6), w3=z(2, 8, 6), offsets=off(3)), **kw))


def backward(**kw):
    return ds.moe_gated_matmul_backward(**dict(dict(dh=z(4, 6), x=z(4, 8), w1=z(2, 8, 6), w3=z(2, 8, 6), saved=z(2, 4, 6, dtype=F32), offsets=off(3)), **kw))


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("case", FORWARD)
def test_both_refuse(case, call):
    with pytest.raises(ds.DsmoeError) as e:
        call(**FORWARD[case])
    assert e.value.status == -1 and "moe_gated_matmul" in str(e.value)


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("case", SIZES)
def test_sizes_beyond_32_bits_are_refused(case, call):
    with pytest.raises(ds.DsmoeError, match="2\\^31") as e:
        call(**SIZES[case])
    assert e.value.status == -1


@pytest.mark.parametrize("kw", [dict(dh=z(4, 5)), dict(dh=z(5, 6)), dict(dh=z(4, 6, dtype=F32)), dict(dh=z(6, 4).t()), dict(saved=z(2, 4, 6)), dict(saved=z(4, 12, dtype=F32)),
                                dict(saved=z(2, 4, 7, dtype=F32)[:, :, :6])], ids=range(7))
def test_backward_refuses(kw):
    with pytest.raises(ds.DsmoeError) as e:
        backward(**kw)
    assert e.value.status == -1 and "moe_gated_matmul_backward" in str(e.value) and "GPU" not in str(e.value)


P = 1 << 20  # an address that nothing reads: every call below is refused
ARGS = dict(rows=10, groups=2, k=64, n=32, dtype=1, activation=0, x_stride=64, w_group_stride=64 * 32, w_row_stride=32, h_stride=32)
BAD = [dict(rows=-1), dict(groups=0), dict(k=0), dict(n=0), dict(dtype=3), dict(dtype=-1), dict(activation=2), dict(activation=-1), dict(x_stride=-1),
       dict(w_group_stride=-1), dict(w_row_stride=-1), dict(h_stride=-1), dict(rows=(1 << 23) + 1), dict(groups=1 << 17), dict(k=(1 << 24) + 1),
       dict(n=(1 << 24) + 1), dict(rows=1 << 23, n=1 << 24, h_stride=1 << 24)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_boundary(kw):
    a = ops._GatedArgs(**dict(ARGS, **kw))
    assert _lib.moe_gated_matmul(a, P, P, P, P, P, P, None, None) == -1
    assert _lib.moe_gated_matmul_backward(a, P, P, P, P, P, P, P, P, P, P, None) == -1
    if "h_stride" not in kw or len(kw) > 1:
        assert _lib.dsmoe_gated_workspace_bytes(a) == 0 and _lib.dsmoe_gated_backward_workspace_bytes(a) == 0


def test_boundary_of_one_direction():
    short = ops._GatedArgs(**dict(ARGS, h_stride=31))  # rows of h would overlap; rows of dh may
    assert _lib.moe_gated_matmul(short, P, P, P, P, P, P, None, None) == -1
    wide = ops._GatedArgs(**dict(ARGS, rows=1 << 23, k=1 << 24, x_stride=1 << 24))  # dx has more tiles than h
    assert _lib.moe_gated_matmul_backward(wide, P, P, P, P, P, P, P, P, P, P, None) == -1
    large = ops._GatedArgs(**dict(ARGS, k=1 << 24, n=1 << 24, w_row_stride=1 << 24))  # and so have the weights
    assert _lib.moe_gated_matmul_backward(large, P, P, P, P, P, P, P, P, P, P, None) == -1


def test_pointers():
    a, none = ops._GatedArgs(**ARGS), ops._GatedArgs(**dict(ARGS, groups=2))
    good = [P, P, P, P, P, P, None]
    for i in (0, 1, 2, 3, 4):
        p = list(good)
        p[i] = None
        assert _lib.moe_gated_matmul(a, *p, None) == -1, i
    for i, bad in ((0, P + 1), (1, P + 1), (2, P + 1), (4, P + 1), (5, P + 2), (6, P + 128)):
        p = list(good)
        p[i] = bad
        assert _lib.moe_gated_matmul(a, *p, None) == -1, i
    good = [P] * 10
    for i in range(10):
        p = list(good)
        p[i] = None
        assert _lib.moe_gated_matmul_backward(a, *p, None) == -1, i
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9):
        p = list(good)
        p[i] = P + 1
        assert _lib.moe_gated_matmul_backward(a, *p, None) == -1, i
    assert _lib.moe_gated_matmul(None, *good[:7], None) == -1 and _lib.moe_gated_matmul_backward(None, *good, None) == -1
    assert _lib.dsmoe_gated_workspace_bytes(None) == 0 and _lib.dsmoe_gated_backward_workspace_bytes(None) == 0


def test_workspace_sizes():
    """da and db are kept with rows on 16 bytes; few rows split nothing, few tiles of long sums are split."""
    def args(**kw):
        return ops._GatedArgs(**dict(ARGS, **kw))

    assert _lib.dsmoe_gated_backward_workspace_bytes(args(n=33, k=32)) >= 2 * 10 * 40 * 2
    assert _lib.dsmoe_gated_workspace_bytes(args(rows=8, groups=64, k=2048, n=1024)) == 0
    assert _lib.dsmoe_gated_workspace_bytes(args(rows=512, groups=1, k=14336, n=256)) > 0
    assert _lib.dsmoe_gated_workspace_bytes(args(rows=512, groups=1, k=14336, n=256, dtype=0)) == 0


FORWARD_TENSORS = dict(x=z(4, 8), w1=z(2, 8, 6), w3=z(2, 8, 6), out=z(4, 6))
BACKWARD_TENSORS = dict(dh=z(4, 6), x=z(4, 8), w1=z(2, 8, 6), w3=z(2, 8, 6), saved=z(2, 4, 6, dtype=F32))


@pytest.mark.parametrize("call,tensors,name", [(c, t, n) for c, t in ((forward, FORWARD_TENSORS), (backward, BACKWARD_TENSORS)) for n in t])
def test_nothing_is_cut_from_the_graph_in_silence(call, tensors, name):
    """A tensor that needs gradients, or has a tangent, is refused while they are recorded.  (Where they are not, the next check refuses: no GPU here.)"""
    def refusal(change):
        with pytest.raises(ds.DsmoeError) as e:
            call(**{k: change(v.clone()) if k == name else v for k, v in tensors.items()})
        assert e.value.status == -1
        return str(e.value)

    assert "needs gradients" in refusal(lambda t: t.requires_grad_())
    with torch.no_grad():
        assert "on one GPU" in refusal(lambda t: t.requires_grad_())
    assert "on one GPU" in refusal(lambda t: t)
    with torch.autograd.forward_ad.dual_level():
        assert "tangent" in refusal(lambda t: torch.autograd.forward_ad.make_dual(t, torch.ones_like(t)))


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


@pytest.mark.parametrize("call,tensors", [(forward, FORWARD_TENSORS), (backward, BACKWARD_TENSORS)])
def test_streams_of_another_gpu_are_refused(call, tensors, monkeypatch):
    monkeypatch.setattr(ops, "_current_device", lambda: 0)

    def refuse(*_):
        raise AssertionError("the named stream is entered, though it is another GPU's")

    monkeypatch.setattr(torch.cuda, "stream", refuse)
    on = {k: OnGpu0(v) for k, v in tensors.items() if k != "out"}
    with pytest.raises(ds.DsmoeError, match="stream") as e:
        call(**on, offsets=OnGpu0(off(3)), stream=Stream1())
    assert e.value.status == -1
