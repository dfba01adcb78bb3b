"""The operators beside the layer (include/dsmoe.h): products over groups of rows with their gradients, the gated half of a block with its
gradients, products with weights in 8-bit integers and in 4 bits, the norms around a block,
and the norm over all gradients with clipping.  Same names as the C ABI, on torch tensors on the GPU; outputs and workspaces are torch allocations on the stream that
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
_Tensor, _strided = torch.Tensor, torch.strided
GATE_NONE, GATE_TOKEN, GATE_CHANNEL, GATE_FULL = 0, 1, 2, 3


class _BlockNormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "d", "dtype", "gate_kind")]
                + [(n, ctypes.c_float) for n in ("scale", "weight_offset", "eps")] + [("pad", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("x_stride", "branch_stride", "gate_stride", "dy_stride", "dh_stride")])


class _GatedArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("rows", "groups", "k", "n", "dtype", "activation")]
                + [(n, ctypes.c_int64) for n in ("x_stride", "w_group_stride", "w_row_stride", "h_stride")])


class _Int4Args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("rows", "groups", "k", "n", "block", "dtype", "scale_dtype", "pad")]
                + [(n, ctypes.c_int64) for n in ("x_stride", "y_stride", "w_group_stride", "w_row_stride", "scale_group_stride", "scale_row_stride",
                                                 "zero_group_stride", "zero_row_stride")])


class _Grad(ctypes.Structure):  # (seven words of 64 bits, as which the binding fills them in)
    _fields_ = ([(n, ctypes.c_void_p) for n in ("grad", "out")] + [(n, ctypes.c_int64) for n in ("rows", "width", "grad_stride", "out_stride")]
                + [(n, ctypes.c_int32) for n in ("dtype", "pad")])


ACTIVATIONS = {"silu": 0, "gelu_tanh": 1}


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
    gated = ctypes.POINTER(_GatedArgs)
    L.dsmoe_gated_workspace_bytes.argtypes = L.dsmoe_gated_backward_workspace_bytes.argtypes = [gated]
    L.moe_gated_matmul.argtypes = [gated] + [vp] * 8
    L.moe_gated_matmul_backward.argtypes = [gated] + [vp] * 11
    L.moe_grad_norm.argtypes = [vp, i32, vp, vp, vp]
    L.moe_clip_grads.argtypes = [vp, i32, ctypes.c_float, ctypes.c_float, vp, vp, vp]
    L.dsmoe_clip_workspace_bytes.argtypes = []
    L.dsmoe_int4_workspace_bytes.argtypes = [ctypes.POINTER(_Int4Args)]
    L.moe_int4_matmul.argtypes = [ctypes.POINTER(_Int4Args)] + [vp] * 8
    for f in (L.dsmoe_grouped_workspace_bytes, L.dsmoe_grouped_dw_workspace_bytes, L.dsmoe_int8_workspace_bytes, L.dsmoe_block_norm_workspace_bytes,
              L.dsmoe_gated_workspace_bytes, L.dsmoe_gated_backward_workspace_bytes, L.dsmoe_clip_workspace_bytes, L.dsmoe_int4_workspace_bytes):
        f.restype = ctypes.c_size_t
    for f in (L.moe_grouped_matmul, L.moe_grouped_matmul_dw, L.moe_int8_matmul, L.moe_block_norm, L.moe_block_norm_backward, L.moe_gated_matmul,
              L.moe_gated_matmul_backward, L.moe_int4_matmul, L.moe_grad_norm, L.moe_clip_grads):
        f.restype = ctypes.c_int


_declare(_lib)
_CLIP_WORDS = _lib.dsmoe_clip_workspace_bytes() // 4


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


def _gated_args(f, x, w1, w3, offsets, activation):
    if x.dim() != 2 or w1.dim() != 3 or w1.shape != w3.shape:
        _refuse(f, "x must have 2 dimensions, w1 and w3 3 and one shape")
    R, k = x.shape
    G, k_of_w, n = w1.shape
    if R | G | k | n > _INT32_MAX:
        _too_large(f)
    if k != k_of_w:
        _refuse(f, "x must have rows of %d values" % k_of_w)
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or w1.dtype is not x.dtype or w3.dtype is not x.dtype:
        _refuse(f, "x, w1 and w3 must be of one type, bfloat16, float16 or float32")
    if offsets is not None:
        if offsets.dtype is not _INT32 or offsets.dim() != 1 or offsets.shape[0] != G + 1 or not offsets.is_contiguous():
            _bad_offsets(f, G)
    elif G != 1:
        _refuse(f, "several groups need offsets")
    act = ACTIVATIONS.get(activation)
    if act is None:
        _refuse(f, "activation must be one of %s" % ", ".join(ACTIVATIONS))
    x_row, x_value = x.stride()
    w_group, w_row, w_value = w1.stride()
    w3_group, w3_row, w3_value = w3.stride()
    if x_value != 1 and k > 1:
        _no_rows(f, "x")
    if n > 1 and (w_value != 1 or w3_value != 1):
        _no_rows(f, "w1 and w3")
    if w_group != w3_group and G > 1 or w_row != w3_row and k > 1:
        _refuse(f, "w1 and w3 must have the same strides")
    return _GatedArgs(R, G, k, n, dtype, act, x_row, w_group, w_row, n)


def moe_gated_matmul(x, w1, w3, offsets=None, activation="silu", want_saved=False, out=None, stream=None):
    """h[r] = f(x[r] W1[g]) * (x[r] W3[g]) for the rows offsets[g] .. offsets[g + 1] - 1 of each group g: both projections of a block of experts, the
    activation and the product.

    x [rows][k], w1, w3 [groups][k][n] with the same strides, offsets int32 [groups + 1] on the GPU, or None for one group of all rows; bf16, f16 or
    f32; rows of no group come out zero.  activation "silu" (a sigmoid(a)) or "gelu_tanh".  want_saved: (h, saved) with both products as they were
    summed, float32 [2][rows][n], for moe_gated_matmul_backward (rows of no group are left as they were allocated).  out as in moe_grouped_matmul."""
    f = "moe_gated_matmul"
    args = _gated_args(f, x, w1, w3, offsets, activation)
    if (_grad_enabled() and (x.requires_grad or w1.requires_grad or w3.requires_grad or out is not None and out.requires_grad)
            or _forward_mode._current_level >= 0):
        _check_unrecorded(f, x, w1, w3, out)
    device = x.get_device()
    if device < 0 or w1.get_device() != device or w3.get_device() != device or offsets is not None and offsets.get_device() != device:
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_gated_matmul(x, w1, w3, offsets, activation, want_saved, out)
    R, n = args.rows, args.n
    given = out
    if out is None:
        out = x.new_empty(R, n)
    else:
        _check_out(out, (R, n), x, f)
        if R > 1:
            args.h_stride = out.stride(0)
    saved = torch.empty((2, R, n), dtype=torch.float32, device=x.device) if want_saved else None
    size = _lib.dsmoe_gated_workspace_bytes(args)
    workspace = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    rc = _lib.moe_gated_matmul(args, x.data_ptr(), w1.data_ptr(), w3.data_ptr(), None if offsets is None else offsets.data_ptr(), out.data_ptr(),
                               saved.data_ptr() if want_saved else None, workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    if given is not None:
        _written(given)
    return (out, saved) if want_saved else out


def moe_gated_matmul_backward(dh, x, w1, w3, saved, offsets=None, activation="silu", stream=None):
    """Gradients of moe_gated_matmul from that of h: a dict of dx, dw1 and dw3.  The other arguments are those of the forward call, saved what it
    returned with want_saved.  Rows of no group get a dx of zeros, groups without rows gradients of zeros."""
    f = "moe_gated_matmul_backward"
    args = _gated_args(f, x, w1, w3, offsets, activation)
    R, n = args.rows, args.n
    if dh.shape != (R, n) or dh.dtype is not x.dtype:
        _refuse(f, "dh must be [%d][%d], of x's type" % (R, n))
    if saved.shape != (2, R, n) or saved.dtype is not torch.float32 or not saved.is_contiguous():
        _refuse(f, "saved must be float32 [2][%d][%d], contiguous" % (R, n))
    args.h_stride, dh_value = dh.stride()
    if dh_value != 1 and n > 1:
        _no_rows(f, "dh")
    if (_grad_enabled() and (x.requires_grad or w1.requires_grad or w3.requires_grad or dh.requires_grad or saved.requires_grad)
            or _forward_mode._current_level >= 0):
        _check_unrecorded(f, x, w1, w3, dh, saved)
    device = x.get_device()
    if (device < 0 or w1.get_device() != device or w3.get_device() != device or dh.get_device() != device or saved.get_device() != device
            or offsets is not None and offsets.get_device() != device):
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_gated_matmul_backward(dh, x, w1, w3, saved, offsets, activation)
    dx, dw1, dw3 = x.new_empty(R, args.k), x.new_empty(w1.shape), x.new_empty(w1.shape)
    size = _lib.dsmoe_gated_backward_workspace_bytes(args)
    workspace = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    rc = _lib.moe_gated_matmul_backward(args, dh.data_ptr(), x.data_ptr(), w1.data_ptr(), w3.data_ptr(), saved.data_ptr(),
                                        None if offsets is None else offsets.data_ptr(), dx.data_ptr(), dw1.data_ptr(), dw3.data_ptr(),
                                        workspace.data_ptr() if size else None, _raw_stream(device))
    if rc:
        _failed(rc, f)
    return {"dx": dx, "dw1": dw1, "dw3": dw3}


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


def moe_int4_matmul(x, w, w_scale, w_zero=None, offsets=None, block=128, out=None, stream=None):
    """y[r][c] = sum over k of x[r][k] (q[g][c][k] - z[g][c][k // block]) s[g][c][k // block]: products with weights in 4 bits, a scale (and a zero point) for
    each block of an output channel's weights.

    x [rows][k] bf16, f16 or f32; w uint8 [groups][n][(k + 1) // 2], the weight of an even k in a byte's low half, of an odd one in its high half;
    w_scale [groups][n][ceil(k / block)] of x's type or float32; w_zero uint8 of that shape, or None for 8 everywhere; block a power of two
    from 32 on; offsets int32 [groups + 1] on the GPU, or None for one group of all rows.  y has x's type.  Weights whose rows start on
    16 bytes are faster.  Few rows are fast in 16-bit types only, and slow if many of their outputs are infinite or
    NaN.  out as in moe_grouped_matmul."""
    f = "moe_int4_matmul"
    if x.dim() != 2 or w.dim() != 3:
        _refuse(f, "x must have 2 dimensions and w 3")
    R, k = x.shape
    G, n, row_bytes = w.shape
    if R | G | k | n > _INT32_MAX:
        _too_large(f)
    if row_bytes != (k + 1) // 2:
        _refuse(f, "w must have rows of %d bytes, for the %d values of x's" % ((k + 1) // 2, k))
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or w.dtype is not torch.uint8:
        _refuse(f, "x must be bfloat16, float16 or float32 and w uint8")
    if type(block) is not int or not 32 <= block <= 1 << 30 or block & block - 1:
        _refuse(f, "block must be a power of two from 32 on")
    blocks = -(-k // block)
    if w_scale.dtype is not torch.float32 and w_scale.dtype is not x.dtype or w_scale.shape != (G, n, blocks):
        _refuse(f, "w_scale must be [%d][%d][%d] of x's type or float32" % (G, n, blocks))
    z_group = z_row = 0
    if w_zero is not None:
        if w_zero.dtype is not torch.uint8 or w_zero.shape != (G, n, blocks):
            _refuse(f, "w_zero must be uint8 [%d][%d][%d]" % (G, n, blocks))
        z_group, z_row, z_value = w_zero.stride()
        if z_value != 1 and blocks > 1:
            _no_rows(f, "w_zero")
    if offsets is not None:
        if offsets.dtype is not _INT32 or offsets.dim() != 1 or offsets.shape[0] != G + 1 or not offsets.is_contiguous():
            _bad_offsets(f, G)
    elif G != 1:
        _refuse(f, "several groups need offsets")
    x_row, x_value = x.stride()
    w_group, w_row, w_value = w.stride()
    s_group, s_row, s_value = w_scale.stride()
    if x_value != 1 and k > 1:
        _no_rows(f, "x")
    if w_value != 1 and row_bytes > 1:
        _no_rows(f, "w")
    if s_value != 1 and blocks > 1:
        _no_rows(f, "w_scale")
    if (_grad_enabled() and (x.requires_grad or w_scale.requires_grad or out is not None and out.requires_grad)
            or _forward_mode._current_level >= 0):
        _check_unrecorded(f, x, w_scale, out)
    device = x.get_device()
    if (device < 0 or w.get_device() != device or w_scale.get_device() != device or w_zero is not None and w_zero.get_device() != device
            or offsets is not None and offsets.get_device() != device):
        _not_one_gpu(f)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_int4_matmul(x, w, w_scale, w_zero, offsets, block, out)
    given = out
    if out is None:
        out, y_row = x.new_empty(R, n), n
    else:
        _check_out(out, (R, n), x, f)
        y_row = out.stride(0) if R > 1 else n
    args = _Int4Args(R, G, k, n, block, dtype, _DTYPES[w_scale.dtype], 0, x_row, y_row, w_group, w_row, s_group, s_row, z_group, z_row)
    size = _lib.dsmoe_int4_workspace_bytes(args)
    workspace = w.new_empty(size) if size else None
    rc = _lib.moe_int4_matmul(args, x.data_ptr(), w.data_ptr(), w_scale.data_ptr(), None if w_zero is None else w_zero.data_ptr(),
                              None if offsets is None else offsets.data_ptr(), out.data_ptr(), workspace.data_ptr() if size else None,
                              _raw_stream(device))
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


def _rows_of(f, name, t, out):
    """(rows, width, stride, stride of out): what the library takes a tensor as, and another one that is written value for value."""
    if t.numel() == 0:
        return 1, 0, 0, 0
    dims = sorted(((s, o, n) for n, s, o in zip(t.shape, t.stride(), out.stride()) if n > 1), reverse=True)
    merged = []
    for s, o, n in dims:  # (s, o: strides; an outer dimension that goes on where the inner one ends is one with it)
        if merged and merged[-1][0] == s * n and merged[-1][1] == o * n:
            merged[-1] = (s, o, merged[-1][2] * n)
        else:
            merged.append((s, o, n))
    if not merged:
        return 1, t.numel(), 0, 0
    if len(merged) > 2 or merged[-1][:2] != (1, 1):
        _refuse(f, "%s: gradients must be dense, or rows of values next to each other" % name)
    if len(merged) == 1:
        return 1, merged[0][2], 0, 0
    (s, o, rows), (_, _, width) = merged
    if o < width:
        _refuse(f, "%s: rows that are written must not overlap" % name)
    return rows, width, s, o


def _no_tensor(f, name):
    """(Without this a gradient that is None, as of a parameter that took no part, would end in an AttributeError.)"""
    _refuse(f, "%s must be a list of tensors, dense ones; leave out what has no gradient" % name)


def _grads(f, grads, out):
    """The library's array of the tensors, and their GPU."""
    if not isinstance(grads, (list, tuple)) or not grads:
        _refuse(f, "grads must be a list of tensors, of at least one")
    if len(grads) > 1 << 20:
        _refuse(f, "at most 2^20 gradients")
    if out is not grads:
        if not isinstance(out, (list, tuple)) or len(out) != len(grads):
            _refuse(f, "out must be a list of as many tensors as grads")
    device, elsewhere, fields = None, False, []
    recorded = _grad_enabled() or _forward_mode._current_level >= 0
    for i, (t, o) in enumerate(zip(grads, out)):
        if not isinstance(t, _Tensor) or t.layout is not _strided:
            _no_tensor(f, "grads")
        if o is not t and (not isinstance(o, _Tensor) or o.layout is not _strided):
            _no_tensor(f, "out")
        dtype = _DTYPES.get(t.dtype)
        if dtype is None:
            _refuse(f, "gradients must be bfloat16, float16 or float32")
        if o is not t and (o.shape != t.shape or o.dtype is not t.dtype):
            _refuse(f, "out[%d] must have its gradient's shape and type" % i)
        if recorded and (t.requires_grad or o.requires_grad or _forward_mode._current_level >= 0):
            _check_unrecorded(f, t, o)
        rows, width, row, out_row = (1, t.numel(), 0, 0) if t.is_contiguous() and o.is_contiguous() else _rows_of(f, "grads[%d]" % i, t, o)
        if device is None:
            device = t.get_device()
        if t.get_device() != device or o is not t and o.get_device() != device:
            elsewhere = True
        fields += (t.data_ptr(), o.data_ptr(), rows, width, row, out_row, dtype)  # (dtype and pad: one of the seven words)
    return fields, device, elsewhere or device < 0


def _array_of(f, fields, elsewhere):
    if elsewhere:
        _not_one_gpu(f)
    return (ctypes.c_int64 * len(fields))(*fields)


def moe_grad_norm(grads, stream=None):
    """The norm over all gradients together, sqrt(sum of all squares), as a float32 tensor without dimensions; squares and sums are in 64 bits.

    grads: a list of tensors on one GPU, bf16, f16 or f32 in any mixture, each dense or rows of values next to each other."""
    f = "moe_grad_norm"
    fields, device, elsewhere = _grads(f, grads, grads)
    array = _array_of(f, fields, elsewhere)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_grad_norm(grads)
    norm = grads[0].new_empty((), dtype=torch.float32)
    workspace = norm.new_empty(_CLIP_WORDS)
    rc = _lib.moe_grad_norm(array, len(grads), norm.data_ptr(), workspace.data_ptr(), _raw_stream(device))
    if rc:
        _failed(rc, f)
    return norm


def moe_clip_grads(grads, max_norm, eps=1e-6, out=None, stream=None):
    """(clipped, norm): each gradient times min(1, max_norm / (norm + eps)), with the norm of moe_grad_norm.

    out: the tensors that are written and returned, of the gradients' shapes and types; `grads` itself to clip in place; None for new ones.  They must
    overlap neither each other nor (but for its own) a gradient.  Nothing waits for the GPU: an infinity or NaN shows in norm."""
    f = "moe_clip_grads"
    if not max_norm >= 0 or not eps >= 0:
        _refuse(f, "max_norm and eps must not be negative")
    given = out
    fields, device, elsewhere = _grads(f, grads, grads if out is None else out)
    if given is not None and len(set(fields[1::7])) != len(grads):
        places = [fields[i + 1] for i in range(0, len(fields), 7) if fields[i + 3]]  # (of a width; empty tensors lie nowhere)
        if len(set(places)) != len(places):
            _refuse(f, "out must not hold a tensor twice")
    array = _array_of(f, fields, elsewhere)
    if stream is not None or device != _current_device():
        with _entered(f, device, stream):
            return moe_clip_grads(grads, max_norm, eps, given)
    if given is None:
        out = [torch.empty_like(t) for t in grads]  # (on the stream that the call runs on)
        array = _array_of(f, *_grads(f, grads, out)[::2])
    norm = grads[0].new_empty((), dtype=torch.float32)
    workspace = norm.new_empty(_CLIP_WORDS)
    rc = _lib.moe_clip_grads(array, len(grads), max_norm, eps, norm.data_ptr(), workspace.data_ptr(), _raw_stream(device))
    if rc:
        _failed(rc, f)
    if given is not None:
        for t in given:
            _written(t)
    return out, norm
