"""CPU: calls of the gradients' norm and clipping that do not fit are refused before anything is launched, in the Python binding and at the C boundary."""
import pytest
import torch

import paper_2508_18376_amd as ds
from paper_2508_18376_amd import operators as ops
from paper_2508_18376_amd.binding import _lib

F32 = torch.float32


def z(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


BOTH = {
    "no tensors": [],
    "no list": z(4),
    "integers": [z(4), z(4, dtype=torch.int32)],
    "64-bit values": [z(4, dtype=torch.float64)],
    "gaps between values": [z(8)[::2]],
    "gaps between values of rows": [z(4, 8)[:, ::2]],
    "gaps in three dimensions": [z(4, 6, 8)[:, :3, :5]],
    "one value again and again": [z(1).expand(5)],
    "not on a GPU": [z(4)],
}


@pytest.mark.parametrize("call", [ds.moe_grad_norm, lambda g: ds.moe_clip_grads(g, 1.0), lambda g: ds.moe_clip_grads(g, 1.0, out=g)])
@pytest.mark.parametrize("case", BOTH)
def test_both_refuse(case, call):
    with pytest.raises(ds.DsmoeError) as e:
        call(BOTH[case])
    assert e.value.status == -1 and ("one GPU" in str(e.value)) == (case == "not on a GPU")


@pytest.mark.parametrize("kw", [dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1e-6), dict(eps=float("nan")), dict(out=[]), dict(out=[z(4)]),
                                dict(out=[z(4), z(2, 4)]), dict(out=[z(4), z(3, 2, dtype=torch.bfloat16)]), dict(out=z(4)), dict(out=[z(4), z(1, 2).expand(3, 2)]),
                                dict(out=[z(4), z(6)[:4].unfold(0, 2, 1)])], ids=range(11))
def test_clipping_refuses(kw):
    with pytest.raises(ds.DsmoeError) as e:
        ds.moe_clip_grads(**dict(dict(grads=[z(4), z(3, 2)], max_norm=1.0), **kw))
    assert e.value.status == -1 and "moe_clip_grads" in str(e.value) and "GPU" not in str(e.value)


def test_one_place_for_two():
    t = z(4)
    with pytest.raises(ds.DsmoeError, match="twice"):
        ds.moe_clip_grads([z(4), z(4)], 1.0, out=[t, t])


def test_nothing_is_cut_from_the_graph_in_silence():
    leaf = z(4).requires_grad_()
    for call in (lambda: ds.moe_grad_norm([z(4), leaf]), lambda: ds.moe_clip_grads([z(4), leaf], 1.0), lambda: ds.moe_clip_grads([z(4)], 1.0, out=[leaf])):
        with pytest.raises(ds.DsmoeError, match="needs gradients"):
            call()
        with torch.no_grad(), pytest.raises(ds.DsmoeError, match="one GPU"):
            call()
    with torch.autograd.forward_ad.dual_level(), pytest.raises(ds.DsmoeError, match="tangent"):
        ds.moe_grad_norm([torch.autograd.forward_ad.make_dual(z(4), z(4))])


@pytest.mark.parametrize("shape,stride,out,want", [
    ((3, 4), (4, 1), (4, 1), (1, 12, 0, 0)), ((3, 4), (7, 1), (7, 1), (3, 4, 7, 7)), ((3, 4), (1, 3), (1, 3), (1, 12, 0, 0)), ((2, 3, 4), (12, 4, 1), (24, 8, 1), (6, 4, 4, 8)),
    ((2, 3, 4), (30, 10, 1), (12, 4, 1), (6, 4, 10, 4)), ((2, 1, 4), (9, 77, 1), (4, 4, 1), (2, 4, 9, 4)), ((1, 1), (5, 9), (3, 2), (1, 1, 0, 0)), ((5,), (1,), (1,), (1, 5, 0, 0)),
    ((4, 2, 3), (3, 12, 1), (3, 12, 1), (1, 24, 0, 0)), ((0, 3), (9, 1), (3, 1), (1, 0, 0, 0))])
def test_tensors_as_rows(shape, stride, out, want):
    t, o = (torch.empty(200).as_strided(shape, s) for s in (stride, out))
    assert ops._rows_of("f", "t", t, o) == want


P = 1 << 20  # an address that nothing reads: every call below is refused
GRAD = dict(grad=P, out=P, rows=2, width=10, grad_stride=12, out_stride=12, dtype=0, pad=0)


def array(**kw):
    return (ops._Grad * 2)(ops._Grad(**GRAD), ops._Grad(**dict(GRAD, **kw)))


BAD = [dict(grad=None), dict(grad=P + 2), dict(rows=-1), dict(rows=1 << 31), dict(width=-1), dict(width=1 << 31), dict(rows=1, width=(1 << 40) + 1), dict(grad_stride=-1),
       dict(dtype=3), dict(dtype=-1), dict(rows=1 << 30, width=1 << 30)]
BAD_OUT = [dict(out=None), dict(out=P + 2), dict(out_stride=9), dict(out_stride=13), dict(grad_stride=10)]


@pytest.mark.parametrize("kw", BAD + BAD_OUT, ids=str)
def test_boundary(kw):
    assert _lib.moe_clip_grads(array(**kw), 2, 1.0, 1e-6, P, P, None) == -1
    if kw in BAD:
        assert _lib.moe_grad_norm(array(**kw), 2, P, P, None) == -1


def test_boundary_of_the_call():
    good = array()
    for count, norm, work in ((0, P, P), (-1, P, P), ((1 << 20) + 1, P, P), (2, None, P), (2, P + 2, P), (2, P, None), (2, P, P + 128)):
        assert _lib.moe_clip_grads(good, count, 1.0, 1e-6, norm, work, None) == -1 and _lib.moe_grad_norm(good, count, norm, work, None) == -1
    assert _lib.moe_clip_grads(None, 1, 1.0, 1e-6, P, P, None) == -1 and _lib.moe_grad_norm(None, 1, P, P, None) == -1
    for max_norm, eps in ((-1.0, 0.0), (float("nan"), 0.0), (1.0, -1.0), (1.0, float("nan"))):
        assert _lib.moe_clip_grads(good, 2, max_norm, eps, P, P, None) == -1
    assert _lib.dsmoe_clip_workspace_bytes() >= 8
