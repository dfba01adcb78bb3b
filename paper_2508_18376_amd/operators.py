"""The operators beside the layer (include/dsmoe.h): products over groups of rows with their gradients, products in 8-bit integers, and the
norms around a block.  Same names as the C ABI, on torch tensors on the GPU; outputs and workspaces are torch allocations on the stream that
the call runs on (the current one, or `stream`).  A call that does not fit its tensors raises DsmoeError before anything is launched.

Nothing is recorded for automatic differentiation: the gradients are operators of their own.  While gradients are being recorded, tensors that need them
(or have a forward-mode tangent) are refused, because the result would look like a constant.  Call inside torch.no_grad(), or from the
forward and backward of a torch.autograd.Function, where recording is off."""
from __future__ import annotations

import ctypes
import types

import torch
from torch.autograd import forward_ad

from .binding import DsmoeError, _lib, _raw_stream

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_EINVAL, _EHIP = -1, -4
_INT32, _INT32_MAX = torch.int32, (1 << 31) - 1
GATE_NONE, GATE_TOKEN, GATE_CHANNEL, GATE_FULL = 0, 1, 2, 3


class _BlockNormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "d", "dtype", "gate_kind")]
                + [(n, ctypes.c_float) for n in ("scale", "weight_offset", "eps")] + [("pad", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("x_stride", "branch_stride", "gate_stride", "dy_stride", "dh_stride")])


def _declare(L):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    args = ctypes.POINTER(_BlockNormArgs)
    L.moe_grouped_matmul.argtypes = [vp, i64, vp, i64, i64, vp, i32, i32, i32, i32, i32, i32, vp, i64, vp, vp]
    L.dsmoe_grouped_workspace_bytes.argtypes = [i32] * 6
    L.dsmoe_grouped_dw_workspace_bytes.argtypes = [i32] * 5
    L.moe_grouped_matmul_dw.argtypes = [vp, i64, vp, i64, vp, i32, i32, i32, i32, i32, vp, i64, i64, vp, vp]
    L.dsmoe_int8_workspace_bytes.argtypes = [i32] * 4
    L.moe_int8_matmul.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i32, i32, i32, i32, i32, vp, i64, vp, vp]
    L.moe_block_norm.argtypes = [args] + [vp] * 9
    L.dsmoe_block_norm_workspace_bytes.argtypes = [args]
    L.moe_block_norm_backward.argtypes = [args] + [vp] * 15
    for f in (L.dsmoe_grouped_workspace_bytes, L.dsmoe_grouped_dw_workspace_bytes, L.dsmoe_int8_workspace_bytes, L.dsmoe_block_norm_workspace_bytes):
        f.restype = ctypes.c_size_t
    for f in (L.moe_grouped_matmul, L.moe_grouped_matmul_dw, L.moe_int8_matmul, L.moe_block_norm, L.moe_block_norm_backward):
        f.restype = ctypes.c_int


_declare(_lib)


def _refuse(where: str, what: str) -> None:
    raise DsmoeError(_EINVAL, "%s: %s;" % (where, what))


def _failed(rc: int, where: str) -> None:
    e = DsmoeError(rc, where)
    if rc == _EHIP:
        e.args = (e.args[0] + " hipError=%d" % _lib.dsmoe_last_hip_error(None),)
    raise e


# A call on a few rows takes less time on the GPU than here (one token on 64 experts of 2048 x 1024: 8 us), so the checks below read each
# property of a tensor once and make no objects or texts unless they refuse.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _no_rows(where, name):
    _refuse(where, "%s: the values of a row must be contiguous" % name)


def _entered(where, device, stream):
    """The device, and where the call names a stream that stream, made current: allocations then belong to it."""
    if stream is None:
        return torch.cuda.device(device)
    if stream.device.index != device:
        _refuse(where, "stream must be of the tensors' GPU")
    return torch.cuda.stream(stream)


def _not_one_gpu(where):
    _refuse(where, "all tensors must be on one GPU")


def _too_large(where):
    """Sizes go to the library in 32 bits, where larger ones would come out as others.  (Or-ed together they pass the limit if one does.)"""
    _refuse(where, "no dimension may pass 2^31 - 1")


# The calls themselves ask what can be asked in an expression, and come to a function only where that says so (16 rows on 8 experts of 128 x 256: 8.0 us a
# call with the checks of devices, streams, offsets and recording as functions that take the tensors, 7.7 like this).
_grad_enabled = torch.is_grad_enabled
# holds the depth of forward-mode differentiation, below zero without it; where torch does not say, the tensors are asked
_forward_mode = forward_ad if hasattr(forward_ad, "_current_level") else types.SimpleNamespace(_current_level=0)


def _check_unrecorded(where, *tensors) -> None:
    """Refuses tensors whose gradients or tangents the call would have to pass on (see the module's docstring)."""
    for t in tensors:
        if t is not None and t.requires_grad and _grad_enabled():
            _refuse(where, "an input needs gradients, which this call does not record: call it inside torch.no_grad() or a torch.autograd.Function")
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            _refuse(where, "an input has a forward-mode tangent, which this call does not pass on")


def _bad_offsets(where, groups):
    _refuse(where, "offsets must be int32 [%d], contiguous" % (groups + 1))


def _check_out(out, shape, like, where) -> None:
    if out.shape != shape or out.dtype != like.dtype or out.device != like.device:
        _refuse(where, "out must be %s %s on the inputs' device" % (list(shape), like.dtype))
    if shape[-1] > 1 and out.stride(-1) != 1:
        _no_rows(where, "out")


def _written(out) -> None:
    """The caller's `out` has other values now: a graph that kept the old ones for a gradient has to notice.  (Inference tensors are in no graph.)"""
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)


def moe_grouped_matmul(x, w, offsets, w_transposed=False, out=None, stream=None):
    """y[r] = x[r] W[g], or x[r] W[g]^T with w_transposed, for the rows offsets[g] .. offsets[g + 1] - 1 of each group g.

    x [rows][k] ([rows][n] with w_transposed), w [groups][k][n], offsets int32 [groups + 1] on the GPU; bf16, f16 or f32.  Rows of no group
    (before the first offset, from the last one on) come out zero.  Rows and weights may be strided, the values of a row are contiguous.  out, if
    given, is written and returned: it may be strided too, and must not overlap the inputs."""
    f = "moe_grouped_matmul"
    if x.dim() != 2 or w.dim() != 3:
        _refuse(f, "x must have 2 dimensions and w 3")
    R, K = x.shape
    G, k, n = w.shape
    if R | G | k | n > _INT32_MAX:
        _too_large(f)
    N = n
    if w_transposed:
        N, k_of_x = k, n
    else:
        k_of_x = k
    if K != k_of_x:
        _refuse(f, "x must have rows of %d values" % k_of_x)
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or w.dtype is not x.dtype:
        _refuse(f, "x and w must be of one type, bfloat16, float16 or float32")
    if offsets.dtype is not _INT32 or offsets.dim() != 1 or offsets.shape[0] != G + 1 or not offsets.is_contiguous():
        _bad_offsets(f, G)
    x_row, x_value = x.stride()
    w_group, w_row, w_value = w.stride()
    if x_value != 1 and K > 1:
        _no_rows(f, "x")
    if w_value != 1 and n > 1:
        _no_rows(f, "w")
    if _grad_enabled() and (x.requires_grad or w.requires_grad or out is not None and out.requires_grad) or _forward_mode._current_level >= 0:
        _check_unrecorded(f, x, w, out)
    device = x.get_device()
    if device < 0 or w.get_device() != device or offsets.get_device() != device:
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_grouped_matmul(x, w, offsets, w_transposed, out)
    given = out
    if out is None:
        out, y_row = x.new_empty(R, N), N
    else:
        _check_out(out, (R, N), x, f)
        y_row = out.stride(0) if R > 1 else N
    transposed = 1 if w_transposed else 0
    size = _lib.dsmoe_grouped_workspace_bytes(R, G, k, n, transposed, dtype)
    workspace = offsets.new_empty(size // 4) if size else None
    rc = _lib.moe_grouped_matmul(x.data_ptr(), x_row, w.data_ptr(), w_group, w_row, offsets.data_ptr(), R, G, k, n, transposed, dtype,
                                 out.data_ptr(), y_row, workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    if given is not None:
        _written(given)
    return out


def moe_grouped_matmul_dw(x, dy, offsets, out=None, stream=None):
    """dw[g] = sum over the rows of group g of x[r]^T dy[r]: the weights' gradient of moe_grouped_matmul.

    x [rows][k], dy [rows][n], offsets int32 [groups + 1] on the GPU; returns [groups][k][n], zeros for a group without rows.  out as in
    moe_grouped_matmul."""
    f = "moe_grouped_matmul_dw"
    if x.dim() != 2 or dy.dim() != 2 or offsets.dim() != 1 or offsets.shape[0] < 2:
        _refuse(f, "x and dy must have 2 dimensions, offsets 1")
    R, k = x.shape
    rows, n = dy.shape
    G = offsets.shape[0] - 1
    if R | G | k | n > _INT32_MAX:
        _too_large(f)
    if rows != R:
        _refuse(f, "x and dy must have the same rows")
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or dy.dtype is not x.dtype:
        _refuse(f, "x and dy must be of one type, bfloat16, float16 or float32")
    if offsets.dtype is not _INT32 or not offsets.is_contiguous():
        _bad_offsets(f, G)
    x_row, x_value = x.stride()
    dy_row, dy_value = dy.stride()
    if x_value != 1 and k > 1:
        _no_rows(f, "x")
    if dy_value != 1 and n > 1:
        _no_rows(f, "dy")
    if _grad_enabled() and (x.requires_grad or dy.requires_grad or out is not None and out.requires_grad) or _forward_mode._current_level >= 0:
        _check_unrecorded(f, x, dy, out)
    device = x.get_device()
    if device < 0 or dy.get_device() != device or offsets.get_device() != device:
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_grouped_matmul_dw(x, dy, offsets, out)
    given = out
    if out is None:
        out, row, group = x.new_empty(G, k, n), n, k * n
    else:
        _check_out(out, (G, k, n), x, f)
        row = out.stride(1) if k > 1 else n
        group = out.stride(0) if G > 1 else (k - 1) * row + n
    size = _lib.dsmoe_grouped_dw_workspace_bytes(R, G, k, n, dtype)
    workspace = offsets.new_empty(size // 4) if size else None
    rc = _lib.moe_grouped_matmul_dw(x.data_ptr(), x_row, dy.data_ptr(), dy_row, offsets.data_ptr(), R, G, k, n, dtype, out.data_ptr(), group, row,
                                    workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    if given is not None:
        _written(given)
    return out


def moe_int8_matmul(x, w, w_scale, offsets=None, out=None, stream=None):
    """y[r][c] = s[r] * w_scale[g][c] * sum over k of q[r][k] w[g][c][k], with s = max|x[r]| * (1 / 127) in fp32 and q = round(x[r] / s) in 8 bits.

    x [rows][k] bf16, f16 or f32; w int8 [groups][n][k]; w_scale float32 [groups][n]; offsets int32 [groups + 1] on the GPU, or None for
    one group of all rows.  y has x's type.  Weights whose rows start on 16 bytes are faster.  out as in moe_grouped_matmul."""
    f = "moe_int8_matmul"
    if x.dim() != 2 or w.dim() != 3:
        _refuse(f, "x must have 2 dimensions and w 3")
    R, k = x.shape
    G, n, k_of_w = w.shape
    if R | G | k | n > _INT32_MAX:
        _too_large(f)
    if k != k_of_w:
        _refuse(f, "x must have rows of %d values" % k_of_w)
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or w.dtype is not torch.int8:
        _refuse(f, "x must be bfloat16, float16 or float32 and w int8")
    if w_scale.dtype is not torch.float32 or w_scale.shape != (G, n):
        _refuse(f, "w_scale must be float32 [%d][%d]" % (G, n))
    if offsets is not None:
        if offsets.dtype is not _INT32 or offsets.dim() != 1 or offsets.shape[0] != G + 1 or not offsets.is_contiguous():
            _bad_offsets(f, G)
    elif G != 1:
        _refuse(f, "several groups need offsets")
    x_row, x_value = x.stride()
    w_group, w_row, w_value = w.stride()
    s_group, s_value = w_scale.stride()
    if x_value != 1 and k > 1:
        _no_rows(f, "x")
    if w_value != 1 and k > 1:
        _no_rows(f, "w")
    if s_value != 1 and n > 1:
        _no_rows(f, "w_scale")
    if _grad_enabled() and (x.requires_grad or w_scale.requires_grad or out is not None and out.requires_grad) or _forward_mode._current_level >= 0:
        _check_unrecorded(f, x, w_scale, out)
    device = x.get_device()
    if device < 0 or w.get_device() != device or w_scale.get_device() != device or offsets is not None and offsets.get_device() != device:
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_int8_matmul(x, w, w_scale, offsets, out)
    given = out
    if out is None:
        out, y_row = x.new_empty(R, n), n
    else:
        _check_out(out, (R, n), x, f)
        y_row = out.stride(0) if R > 1 else n
    size = _lib.dsmoe_int8_workspace_bytes(R, G, k, n)
    workspace = w.new_empty(size) if size else None
    rc = _lib.moe_int8_matmul(x.data_ptr(), x_row, w.data_ptr(), w_group, w_row, w_scale.data_ptr(), s_group,
                              None if offsets is None else offsets.data_ptr(), R, G, k, n, dtype, out.data_ptr(), y_row,
                              workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    if given is not None:
        _written(given)
    return out


def _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps):
    shape, dtype = x.shape, x.dtype
    if len(shape) != 2 or shape[1] < 1 or branch.shape != shape:
        _refuse(f, "x and branch must be [tokens][d], of one shape")
    T, D = shape
    if T | D > _INT32_MAX:
        _too_large(f)
    if branch_weight.dim() != 1 or weight.dim() != 1 or branch_weight.shape[0] != D or weight.shape[0] != D:
        _refuse(f, "branch_weight and weight must be [%d]" % D)
    code = _DTYPES.get(dtype)
    if code is None or branch.dtype is not dtype or branch_weight.dtype is not dtype or weight.dtype is not dtype:
        _refuse(f, "x, branch, gate and the weights must be of one type, bfloat16, float16 or float32")
    kind = gate_row = 0
    if gate is not None:
        gs = gate.shape
        kind = GATE_FULL if gs == shape else GATE_TOKEN if gs == (T, 1) else GATE_CHANNEL
        if kind == GATE_CHANNEL and gs != (1, D):
            _refuse(f, "gate must be [tokens][1], [1][d] or [tokens][d]")
        if gate.dtype is not dtype:
            _refuse(f, "x, branch, gate and the weights must be of one type, bfloat16, float16 or float32")
        gate_row, gate_value = gate.stride()
        if gate_value != 1 and gs[1] > 1:
            _no_rows(f, "gate")
    x_row, x_value = x.stride()
    b_row, b_value = branch.stride()
    if D > 1:
        if x_value != 1 or b_value != 1:
            _no_rows(f, "x and branch")
        if branch_weight.stride()[0] != 1 or weight.stride()[0] != 1:
            _no_rows(f, "branch_weight and weight")
    if not eps >= 0:
        _refuse(f, "eps must not be negative")
    return _BlockNormArgs(T, D, code, kind, scale, weight_offset, eps, 0, x_row, b_row, gate_row)


def moe_block_norm(x, *, branch, branch_weight, weight, gate=None, scale=1.0, weight_offset=0.0, eps=1e-6, want_stats=False, stream=None):
    """(y, h) with y = x + scale * gate * norm(branch) * (branch_weight + weight_offset) and h = norm(y) * (weight + weight_offset), where
    norm(v) = v * rsqrt(mean(v^2) + eps): the norm behind a block, its gate and residual connection, and the norm in front of the next one.

    x, branch [tokens][d]; branch_weight, weight [d]; gate None, [tokens][1], [1][d] or [tokens][d].  want_stats: also the rows' statistics
    (float32 [2][tokens]) for moe_block_norm_backward."""
    f = "moe_block_norm"
    args = _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps)
    if _grad_enabled() and (x.requires_grad or branch.requires_grad or branch_weight.requires_grad or weight.requires_grad
                            or gate is not None and gate.requires_grad) or _forward_mode._current_level >= 0:
        _check_unrecorded(f, x, branch, branch_weight, weight, gate)
    device = x.get_device()
    if (device < 0 or branch.get_device() != device or branch_weight.get_device() != device or weight.get_device() != device
            or gate is not None and gate.get_device() != device):
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_block_norm(x, branch=branch, branch_weight=branch_weight, weight=weight, gate=gate, scale=scale, weight_offset=weight_offset,
                                  eps=eps, want_stats=want_stats)
    T, D = args.tokens, args.d
    y, h = x.new_empty(T, D), x.new_empty(T, D)
    stats = torch.empty((2, T), dtype=torch.float32, device=x.device) if want_stats else None
    rc = _lib.moe_block_norm(args, x.data_ptr(), branch.data_ptr(), branch_weight.data_ptr(), None if gate is None else gate.data_ptr(),
                             weight.data_ptr(), y.data_ptr(), h.data_ptr(), stats.data_ptr() if want_stats else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    return (y, h, stats) if want_stats else (y, h)


def moe_block_norm_backward(dy, dh, x, stats, *, branch, branch_weight, weight, gate=None, scale=1.0, weight_offset=0.0, eps=1e-6, stream=None):
    """Gradients of moe_block_norm from those of y and h: a dict of dx, dbranch, dbranch_weight, dweight and, with a gate, dgate (the gate's
    shape).  The other arguments are those of the forward call, stats what it returned with want_stats."""
    f = "moe_block_norm_backward"
    args = _norm_args(f, x, branch, branch_weight, gate, weight, scale, weight_offset, eps)
    T, D = args.tokens, args.d
    if dy.shape != x.shape or dh.shape != x.shape or dy.dtype is not x.dtype or dh.dtype is not x.dtype:
        _refuse(f, "dy and dh must have x's shape and type")
    if stats.shape != (2, T) or stats.dtype is not torch.float32 or not stats.is_contiguous():
        _refuse(f, "stats must be float32 [2][%d], contiguous" % T)
    args.dy_stride, dy_value = dy.stride()
    args.dh_stride, dh_value = dh.stride()
    if D > 1 and (dy_value != 1 or dh_value != 1):
        _no_rows(f, "dy and dh")
    if _grad_enabled() and (x.requires_grad or dy.requires_grad or dh.requires_grad or stats.requires_grad or branch.requires_grad
                            or branch_weight.requires_grad or weight.requires_grad or gate is not None and gate.requires_grad) or _forward_mode._current_level >= 0:
        _check_unrecorded(f, x, dy, dh, stats, branch, branch_weight, weight, gate)
    device = x.get_device()
    if (device < 0 or dy.get_device() != device or dh.get_device() != device or stats.get_device() != device or branch.get_device() != device
            or branch_weight.get_device() != device or weight.get_device() != device or gate is not None and gate.get_device() != device):
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_block_norm_backward(dy, dh, x, stats, branch=branch, branch_weight=branch_weight, weight=weight, gate=gate, scale=scale,
                                           weight_offset=weight_offset, eps=eps)
    out = {"dx": x.new_empty(T, D), "dbranch": x.new_empty(T, D), "dbranch_weight": x.new_empty(D), "dweight": x.new_empty(D)}
    if gate is not None:
        out["dgate"] = x.new_empty(gate.shape)
    size = _lib.dsmoe_block_norm_workspace_bytes(args)
    workspace = stats.new_empty((size + 3) // 4) if size else None
    rc = _lib.moe_block_norm_backward(args, dy.data_ptr(), dh.data_ptr(), x.data_ptr(), branch.data_ptr(), branch_weight.data_ptr(),
                                      None if gate is None else gate.data_ptr(), weight.data_ptr(), stats.data_ptr(), out["dx"].data_ptr(),
                                      out["dbranch"].data_ptr(), out["dbranch_weight"].data_ptr(), None if gate is None else out["dgate"].data_ptr(),
                                      out["dweight"].data_ptr(), workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    return out
