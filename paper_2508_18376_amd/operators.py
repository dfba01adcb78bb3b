"""The operators beside the layer (include/dsmoe.h): products over groups of rows with their gradients, products in 8-bit integers, and the
norms around a block.  Same names as the C ABI, on torch tensors on the GPU; outputs and workspaces are torch allocations on the stream that
the call runs on (the current one, or `stream`).  A call that does not fit its tensors raises DsmoeError before anything is launched."""
from __future__ import annotations

import ctypes

import torch

from .binding import _NO_SWITCH, DsmoeError, _lib, _raw_stream

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_EINVAL, _EHIP = -1, -4
GATE_NONE, GATE_TOKEN, GATE_CHANNEL, GATE_FULL = 0, 1, 2, 3


class _BlockNormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "d", "dtype", "gate_kind")]
                + [(n, ctypes.c_float) for n in ("scale", "weight_offset", "eps")] + [("pad", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("x_stride", "branch_stride", "gate_stride", "dy_stride", "dh_stride")])


def _declare(L):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    args = ctypes.POINTER(_BlockNormArgs)
    L.moe_grouped_matmul.argtypes = [vp, i64, vp, i64, i64, vp, i32, i32, i32, i32, i32, i32, vp, i64, vp]
    L.moe_grouped_matmul_dw.argtypes = [vp, i64, vp, i64, vp, i32, i32, i32, i32, i32, vp, i64, i64, vp]
    L.dsmoe_int8_workspace_bytes.argtypes = [i32, i32]
    L.moe_int8_matmul.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i32, i32, i32, i32, i32, vp, i64, vp, vp]
    L.moe_block_norm.argtypes = [args] + [vp] * 9
    L.dsmoe_block_norm_workspace_bytes.argtypes = [args]
    L.moe_block_norm_backward.argtypes = [args] + [vp] * 15
    for f in (L.dsmoe_int8_workspace_bytes, L.dsmoe_block_norm_workspace_bytes):
        f.restype = ctypes.c_size_t
    for f in (L.moe_grouped_matmul, L.moe_grouped_matmul_dw, L.moe_int8_matmul, L.moe_block_norm, L.moe_block_norm_backward):
        f.restype = ctypes.c_int


_declare(_lib)


def _need(ok, where: str, what: str) -> None:
    if not ok:
        raise DsmoeError(_EINVAL, "%s: %s;" % (where, what))


def _check(rc: int, where: str) -> None:
    if rc != 0:
        e = DsmoeError(rc, where)
        if rc == _EHIP:
            e.args = (e.args[0] + " hipError=%d" % _lib.dsmoe_last_hip_error(None),)
        raise e


def _rows_ok(t, where, name) -> None:
    """The values of a row lie next to each other."""
    _need(t.shape[-1] <= 1 or t.stride(-1) == 1, where, "%s: the values of a row must be contiguous" % name)


def _on_gpu(where, device, **tensors) -> None:
    for name, t in tensors.items():
        _need(t is None or (t.is_cuda and t.device == device), where, "%s: all tensors must be on one GPU" % name)


def _entered(device, stream):
    """The device, and where the call names a stream that stream, made current: allocations then belong to it."""
    if stream is not None:
        return torch.cuda.stream(stream)
    return _NO_SWITCH if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _check_offsets(offsets, groups, where) -> None:
    _need(offsets.dtype == torch.int32 and offsets.dim() == 1 and offsets.shape[0] == groups + 1 and offsets.is_contiguous(), where,
          "offsets must be int32 [%d], contiguous" % (groups + 1))


def _output(out, shape, like, where):
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    _need(tuple(out.shape) == tuple(shape) and out.dtype == like.dtype and out.device == like.device, where,
          "out must be %s %s on the inputs' device" % (list(shape), like.dtype))
    _rows_ok(out, where, "out")
    return out


def moe_grouped_matmul(x, w, offsets, w_transposed=False, out=None, stream=None):
    """y[r] = x[r] W[g], or x[r] W[g]^T with w_transposed, for the rows offsets[g] .. offsets[g + 1] - 1 of each group g.

    x [rows][k] ([rows][n] with w_transposed), w [groups][k][n], offsets int32 [groups + 1] on the GPU; bf16, f16 or f32.  Rows of no group
    (before the first offset, from the last one on) come out zero.  Rows and weights may be strided, the values of a row are contiguous."""
    f = "moe_grouped_matmul"
    _need(x.dim() == 2 and w.dim() == 3, f, "x must have 2 dimensions and w 3")
    R, G, k, n = x.shape[0], w.shape[0], w.shape[1], w.shape[2]
    K, N = (n, k) if w_transposed else (k, n)
    _need(x.shape[1] == K, f, "x must have rows of %d values" % K)
    _need(x.dtype == w.dtype and x.dtype in _DTYPES, f, "x and w must be of one type, bfloat16, float16 or float32")
    _check_offsets(offsets, G, f)
    _rows_ok(x, f, "x")
    _rows_ok(w, f, "w")
    _on_gpu(f, x.device, x=x, w=w, offsets=offsets)
    with _entered(x.device, stream):
        y = _output(out, (R, N), x, f)
        _check(_lib.moe_grouped_matmul(x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), w.stride(1), offsets.data_ptr(), R, G, k, n,
                                       1 if w_transposed else 0, _DTYPES[x.dtype], y.data_ptr(), max(y.stride(0), N) if R < 2 else y.stride(0),
                                       _raw_stream(x.device.index)), f)
    return y


def moe_grouped_matmul_dw(x, dy, offsets, out=None, stream=None):
    """dw[g] = sum over the rows of group g of x[r]^T dy[r]: the weights' gradient of moe_grouped_matmul.

    x [rows][k], dy [rows][n], offsets int32 [groups + 1] on the GPU; returns [groups][k][n], zeros for a group without rows."""
    f = "moe_grouped_matmul_dw"
    _need(x.dim() == 2 and dy.dim() == 2 and offsets.dim() == 1 and offsets.shape[0] >= 2, f, "x and dy must have 2 dimensions, offsets 1")
    R, k, n, G = x.shape[0], x.shape[1], dy.shape[1], offsets.shape[0] - 1
    _need(dy.shape[0] == R, f, "x and dy must have the same rows")
    _need(x.dtype == dy.dtype and x.dtype in _DTYPES, f, "x and dy must be of one type, bfloat16, float16 or float32")
    _check_offsets(offsets, G, f)
    _rows_ok(x, f, "x")
    _rows_ok(dy, f, "dy")
    _on_gpu(f, x.device, x=x, dy=dy, offsets=offsets)
    with _entered(x.device, stream):
        dw = _output(out, (G, k, n), x, f)
        row = max(dw.stride(1), n) if k < 2 else dw.stride(1)
        group = max(dw.stride(0), (k - 1) * row + n) if G < 2 else dw.stride(0)
        _check(_lib.moe_grouped_matmul_dw(x.data_ptr(), x.stride(0), dy.data_ptr(), dy.stride(0), offsets.data_ptr(), R, G, k, n, _DTYPES[x.dtype],
                                          dw.data_ptr(), group, row, _raw_stream(x.device.index)), f)
    return dw


def moe_int8_matmul(x, w, w_scale, offsets=None, out=None, stream=None):
    """y[r][c] = s[r] * w_scale[g][c] * sum over k of q[r][k] w[g][c][k], with s = max|x[r]| / 127 and q = round(x[r] / s) in 8 bits.

    x [rows][k] bf16, f16 or f32; w int8 [groups][n][k]; w_scale float32 [groups][n]; offsets int32 [groups + 1] on the GPU, or None for
    one group of all rows.  y has x's type.  Weights whose rows start on 16 bytes are faster."""
    f = "moe_int8_matmul"
    _need(x.dim() == 2 and w.dim() == 3, f, "x must have 2 dimensions and w 3")
    R, k, G, n = x.shape[0], x.shape[1], w.shape[0], w.shape[1]
    _need(w.shape[2] == k, f, "x must have rows of %d values" % w.shape[2])
    _need(x.dtype in _DTYPES and w.dtype == torch.int8, f, "x must be bfloat16, float16 or float32 and w int8")
    _need(w_scale.dtype == torch.float32 and tuple(w_scale.shape) == (G, n), f, "w_scale must be float32 [%d][%d]" % (G, n))
    if offsets is not None:
        _check_offsets(offsets, G, f)
    _need(offsets is not None or G == 1, f, "several groups need offsets")
    for name, t in (("x", x), ("w", w), ("w_scale", w_scale)):
        _rows_ok(t, f, name)
    _on_gpu(f, x.device, x=x, w=w, w_scale=w_scale, offsets=offsets)
    with _entered(x.device, stream):
        y = _output(out, (R, n), x, f)
        workspace = torch.empty(_lib.dsmoe_int8_workspace_bytes(R, k), dtype=torch.uint8, device=x.device)
        _check(_lib.moe_int8_matmul(x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), w.stride(1), w_scale.data_ptr(), w_scale.stride(0),
                                    None if offsets is None else offsets.data_ptr(), R, G, k, n, _DTYPES[x.dtype], y.data_ptr(),
                                    max(y.stride(0), n) if R < 2 else y.stride(0), workspace.data_ptr(), _raw_stream(x.device.index)), f)
    return y


def _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps):
    _need(x.dim() == 2 and x.shape[1] > 0 and branch.shape == x.shape, f, "x and branch must be [tokens][d], of one shape")
    T, D = x.shape
    _need(branch_weight.shape == (D,) and weight.shape == (D,), f, "branch_weight and weight must be [%d]" % D)
    kind = GATE_NONE
    if gate is not None:
        _need(gate.dim() == 2 and gate.shape[0] in (1, T) and gate.shape[1] in (1, D), f, "gate must be [tokens][1], [1][d] or [tokens][d]")
        kind = GATE_FULL if gate.shape == x.shape else GATE_TOKEN if gate.shape == (T, 1) else GATE_CHANNEL
        _need(kind != GATE_CHANNEL or gate.shape == (1, D), f, "gate must be [tokens][1], [1][d] or [tokens][d]")
        _rows_ok(gate, f, "gate")
    _need(x.dtype in _DTYPES and all(t is None or t.dtype == x.dtype for t in (branch, branch_weight, gate, weight)), f,
          "x, branch, gate and the weights must be of one type, bfloat16, float16 or float32")
    for name, t in (("x", x), ("branch", branch), ("branch_weight", branch_weight), ("weight", weight)):
        _rows_ok(t, f, name)
    _need(eps >= 0, f, "eps must not be negative")
    return _BlockNormArgs(T, D, _DTYPES[x.dtype], kind, scale, weight_offset, eps, 0, x.stride(0), branch.stride(0), 0 if gate is None else gate.stride(0))


def _ptr(t):
    return None if t is None else t.data_ptr()


def moe_block_norm(x, *, branch, branch_weight, weight, gate=None, scale=1.0, weight_offset=0.0, eps=1e-6, want_stats=False, stream=None):
    """(y, h) with y = x + scale * gate * norm(branch) * (branch_weight + weight_offset) and h = norm(y) * (weight + weight_offset), where
    norm(v) = v * rsqrt(mean(v^2) + eps): the norm behind a block, its gate and residual connection, and the norm in front of the next one.

    x, branch [tokens][d]; branch_weight, weight [d]; gate None, [tokens][1], [1][d] or [tokens][d].  want_stats: also the rows' statistics
    (float32 [2][tokens]) for moe_block_norm_backward."""
    f = "moe_block_norm"
    args = _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps)
    _on_gpu(f, x.device, x=x, branch=branch, branch_weight=branch_weight, gate=gate, weight=weight)
    with _entered(x.device, stream):
        y, h = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(2))
        stats = torch.empty((2, x.shape[0]), dtype=torch.float32, device=x.device) if want_stats else None
        _check(_lib.moe_block_norm(args, x.data_ptr(), branch.data_ptr(), branch_weight.data_ptr(), _ptr(gate), weight.data_ptr(), y.data_ptr(),
                                   h.data_ptr(), _ptr(stats), _raw_stream(x.device.index)), f)
    return (y, h, stats) if want_stats else (y, h)


def moe_block_norm_backward(dy, dh, x, stats, *, branch, branch_weight, weight, gate=None, scale=1.0, weight_offset=0.0, eps=1e-6, stream=None):
    """Gradients of moe_block_norm from those of y and h: a dict of dx, dbranch, dbranch_weight, dweight and, with a gate, dgate (the gate's
    shape).  The other arguments are those of the forward call, stats what it returned with want_stats."""
    f = "moe_block_norm_backward"
    args = _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps)
    _need(dy.shape == x.shape and dh.shape == x.shape and dy.dtype == x.dtype and dh.dtype == x.dtype, f, "dy and dh must have x's shape and type")
    _need(stats.shape == (2, x.shape[0]) and stats.dtype == torch.float32 and stats.is_contiguous(), f, "stats must be float32 [2][%d]" % x.shape[0])
    _rows_ok(dy, f, "dy")
    _rows_ok(dh, f, "dh")
    args.dy_stride, args.dh_stride = dy.stride(0), dh.stride(0)
    _on_gpu(f, x.device, dy=dy, dh=dh, x=x, stats=stats, branch=branch, branch_weight=branch_weight, gate=gate, weight=weight)
    with _entered(x.device, stream):
        def empty(*shape):
            return torch.empty(shape, dtype=x.dtype, device=x.device)

        out = {"dx": empty(*x.shape), "dbranch": empty(*x.shape), "dbranch_weight": empty(x.shape[1]), "dweight": empty(x.shape[1])}
        if gate is not None:
            out["dgate"] = empty(*gate.shape)
        workspace = torch.empty(_lib.dsmoe_block_norm_workspace_bytes(args), dtype=torch.uint8, device=x.device)
        _check(_lib.moe_block_norm_backward(args, dy.data_ptr(), dh.data_ptr(), x.data_ptr(), branch.data_ptr(), branch_weight.data_ptr(), _ptr(gate),
                                            weight.data_ptr(), stats.data_ptr(), out["dx"].data_ptr(), out["dbranch"].data_ptr(),
                                            out["dbranch_weight"].data_ptr(), _ptr(out.get("dgate")), out["dweight"].data_ptr(),
                                            workspace.data_ptr(), _raw_stream(x.device.index)), f)
    return out
