"""CPU: calls of the 4-bit products that do not fit their tensors are refused before anything is launched, in the Python binding and at the C boundary."""
import pytest
import torch

import paper_2508_18376_amd as ds
from paper_2508_18376_amd import operators as ops
from paper_2508_18376_amd.binding import _lib

I32, BF, F32, U8 = torch.int32, torch.bfloat16, torch.float32, torch.uint8
MANY = (1 << 32) + 5


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def off(n):
    return torch.zeros(n, dtype=I32)


def int4(**kw):
    a = dict(x=z(4, 70), w=z(2, 6, 35, dtype=U8), w_scale=z(2, 6, 3), w_zero=z(2, 6, 3, dtype=U8), offsets=off(3), block=32)
    return ds.moe_int4_matmul(**dict(a, **kw))


CASES = {
    "x of 3 dimensions": dict(x=z(1, 4, 70)),
    "w of 2 dimensions": dict(w=z(6, 35, dtype=U8)),
    "rows of w too short": dict(w=z(2, 6, 34, dtype=U8)),
    "rows of w too long": dict(w=z(2, 6, 36, dtype=U8)),
    "w in int8": dict(w=z(2, 6, 35, dtype=torch.int8)),
    "x in int8": dict(x=z(4, 70, dtype=torch.int8)),
    "x in 64 bits": dict(x=z(4, 70, dtype=torch.float64)),
    "block of no power of two": dict(block=48),
    "block too small": dict(block=16, w_scale=z(2, 6, 5), w_zero=None),
    "block of zero": dict(block=0),
    "block of another type": dict(block=32.0),
    "block beyond 32 bits": dict(block=1 << 31, w_scale=z(2, 6, 1), w_zero=None),
    "scales for too few blocks": dict(w_scale=z(2, 6, 2)),
    "scales for too few channels": dict(w_scale=z(2, 5, 3)),
    "scales of another 16-bit type": dict(w_scale=z(2, 6, 3, dtype=torch.float16)),
    "scales in 16 bits for x in 32": dict(x=z(4, 70, dtype=F32)),
    "zero points for too few blocks": dict(w_zero=z(2, 6, 2, dtype=U8)),
    "zero points in int8": dict(w_zero=z(2, 6, 3, dtype=torch.int8)),
    "zero points in bf16": dict(w_zero=z(2, 6, 3)),
    "64-bit offsets": dict(offsets=off(3).long()),
    "offsets too long": dict(offsets=off(4)),
    "groups without offsets": dict(offsets=None),
    "x by columns": dict(x=z(70, 4).t()),
    "w by columns": dict(w=z(2, 35, 6, dtype=U8).transpose(1, 2)),
    "scales by columns": dict(w_scale=z(2, 3, 6).transpose(1, 2)),
    "zero points by columns": dict(w_zero=z(2, 3, 6, dtype=U8).transpose(1, 2)),
    "not on a GPU": dict(),
}


@pytest.mark.parametrize("case", CASES)
def test_refusals(case):
    with pytest.raises(ds.DsmoeError) as e:
        int4(**CASES[case])
    assert e.value.status == -1 and "moe_int4_matmul" in str(e.value) and ("one GPU" in str(e.value)) == (case == "not on a GPU")


@pytest.mark.parametrize("kw", [dict(x=z(1, 70).expand(MANY, 70)), dict(w=z(2, 1, 35, dtype=U8).expand(2, MANY, 35))], ids=["rows", "channels"])
def test_sizes_beyond_32_bits_are_refused(kw):
    with pytest.raises(ds.DsmoeError, match="2\\^31") as e:
        int4(**kw)
    assert e.value.status == -1


@pytest.mark.parametrize("name", ["x", "w_scale", "out"])
def test_nothing_is_cut_from_the_graph_in_silence(name):
    def refusal(change):
        tensors = dict(x=z(4, 70), w_scale=z(2, 6, 3), out=z(4, 6))
        tensors[name] = change(tensors[name])
        with pytest.raises(ds.DsmoeError) as e:
            int4(**tensors)
        return str(e.value)

    assert "needs gradients" in refusal(lambda t: t.requires_grad_())
    with torch.no_grad():
        assert "on one GPU" in refusal(lambda t: t.requires_grad_())
    with torch.autograd.forward_ad.dual_level():
        assert "tangent" in refusal(lambda t: torch.autograd.forward_ad.make_dual(t, torch.ones_like(t)))


P = 1 << 20  # an address that nothing reads: every call below is refused
ARGS = dict(rows=10, groups=2, k=64, n=32, block=32, dtype=1, scale_dtype=1, pad=0, x_stride=64, y_stride=32, w_group_stride=1024, w_row_stride=32,
            scale_group_stride=64, scale_row_stride=2, zero_group_stride=64, zero_row_stride=2)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(groups=0), dict(k=0), dict(n=0), dict(block=16), dict(block=0), dict(block=-32), dict(block=96),
                                dict(block=-(1 << 31)), dict(dtype=3), dict(dtype=-1), dict(scale_dtype=2), dict(dtype=0), dict(scale_dtype=3), dict(x_stride=-1),
                                dict(y_stride=31), dict(w_group_stride=-1), dict(w_row_stride=-1), dict(scale_group_stride=-1), dict(scale_row_stride=-1),
                                dict(zero_group_stride=-1), dict(zero_row_stride=-1), dict(rows=(1 << 23) + 1), dict(groups=1 << 17), dict(k=(1 << 24) + 1),
                                dict(rows=1 << 23, n=1 << 24, y_stride=1 << 24)], ids=str)
def test_boundary(kw):
    assert _lib.moe_int4_matmul(ops._Int4Args(**dict(ARGS, **kw)), P, P, P, P, P, P, None, None) == -1


def test_pointers():
    a, good = ops._Int4Args(**ARGS), [P, P, P, P, P, P]
    for i in (0, 1, 2, 4, 5):  # (the zero points may be missing)
        p = list(good)
        p[i] = None
        assert _lib.moe_int4_matmul(a, *p, None, None) == -1, i
    for i in (0, 2, 5):
        p = list(good)
        p[i] = P + 1
        assert _lib.moe_int4_matmul(a, *p, None, None) == -1, i
    assert _lib.moe_int4_matmul(None, *good, None, None) == -1 and _lib.moe_int4_matmul(a, *good, P + 128, None) == -1


def test_workspace_sizes():
    """Few tiles of long sums are split, and the last ones of many; streams, short sums, many rows and fp32 are not."""
    def size(**kw):
        return _lib.dsmoe_int4_workspace_bytes(ops._Int4Args(**dict(ARGS, **kw)))

    assert size(rows=1, groups=1, k=8192, n=4096) > 0 and size(rows=512, groups=1, k=4096, n=4096) > 0 and size(rows=8300, groups=1, k=2048, n=1808) > 0
    assert size(rows=1, groups=1, k=4096, n=4096) == 0 and size(rows=512, groups=1, k=256, n=4096) == 0 and size(rows=64, groups=8, k=4096, n=1 << 17) == 0
    assert size(rows=1, groups=1, k=4096, n=4096, dtype=0, scale_dtype=0) == 0 and size(rows=-1) == 0 and size(block=48) == 0
    assert _lib.dsmoe_int4_workspace_bytes(None) == 0


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


def test_streams_of_another_gpu_are_refused(monkeypatch):
    monkeypatch.setattr(ops, "_current_device", lambda: 0)

    def refuse(*_):
        raise AssertionError("the named stream is entered, though it is another GPU's")

    monkeypatch.setattr(torch.cuda, "stream", refuse)
    on = dict(x=z(4, 70), w=z(2, 6, 35, dtype=U8), w_scale=z(2, 6, 3), w_zero=z(2, 6, 3, dtype=U8), offsets=off(3))
    with pytest.raises(ds.DsmoeError, match="stream"):
        int4(**{k: OnGpu0(v) for k, v in on.items()}, stream=Stream1())
