"""The operators on rows in device memory (include/gvhot.h) for tensors of torch: shapes, strides and types are read
from the tensors, results that the caller does not pass are allocated, and the kernels go to torch's current stream
of the tensors' GPU.  Rows are 2-D tensors whose last dimension is contiguous; their rows may lie further apart.
No arithmetic happens here.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple, Optional

import torch

from .binding import GV_BF16, GV_F16, GV_F32, GV_I8, GV_OK, GvError, load

__all__ = ["NormRows", "NormGrads", "gv_drop_rows", "gv_norm_rows", "gv_norm_rows_workspace", "gv_norm_rows_backward",
           "gv_quantize_rows", "gv_score_rows"]

_TYPES = {torch.float32: GV_F32, torch.bfloat16: GV_BF16, torch.float16: GV_F16}
_TYPES_AND_BYTES = dict(_TYPES)
_TYPES_AND_BYTES[torch.int8] = GV_I8


class NormRows(NamedTuple):
    """What gv_norm_rows gives; None where it was not asked for."""
    out: torch.Tensor
    scale: Optional[torch.Tensor]  # float32[rows], of an 8-bit out
    sum: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]   # float32[rows]


class NormGrads(NamedTuple):
    x: torch.Tensor
    residual: Optional[torch.Tensor]
    gain: Optional[torch.Tensor]   # float32[cols]


def _refuse(text):
    raise ValueError(text)


def _rows(name, t, like=None, dtype=None):
    """(address, stride) of a matrix of rows, which has to be like another."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        _refuse(f"{name}: a 2-D tensor whose rows are contiguous")
    if like is not None and (t.shape != like.shape or t.device != like.device or t.dtype is not (dtype or like.dtype)):
        _refuse(f"{name}: shape, type or device does not fit")
    rows, cols = t.shape
    return t.data_ptr(), (t.stride(0) if rows > 1 else cols)


def _kind(t, kinds, name):
    if not t.is_cuda:
        _refuse(f"{name}: not in device memory")
    kind = kinds.get(t.dtype)
    if kind is None:
        _refuse(f"{name}: type {t.dtype} is not supported")
    return kind


def _array(name, t, size, dtype, like):
    """Address of a contiguous array of `size` values."""
    if t.dtype is not dtype or t.numel() != size or not t.is_contiguous() or t.device != like.device:
        _refuse(f"{name}: {size} contiguous values of {dtype} on {like.device}")
    return t.data_ptr()


def _call(entry, device, *args):
    stream = torch.cuda.current_stream(device).cuda_stream
    if device.index == torch.cuda.current_device():
        rc = entry(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = entry(*args, stream)
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())


def gv_drop_rows(x, drop, seed, *, first_row=0, out=None):
    """Dropout of rows.  The gradient of x is the same call, with the same drop, seed and first_row, on out's gradient."""
    kind = _kind(x, _TYPES, "x")
    rows, cols = x.shape if x.dim() == 2 else _refuse("x: a 2-D tensor")
    at, stride = _rows("x", x)
    if out is None:
        out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    out_at, out_stride = _rows("out", out, x)
    _call(load().gv_drop_rows, x.device, rows, cols, kind, at, stride, drop, seed, first_row, out_at, out_stride)
    return out


def gv_norm_rows(x, gain, residual=None, *, eps=1e-6, drop=0.0, seed=0, first_row=0, out_type=None, keep_sum=True,
                 keep_rstd=False, out=None, scale=None, sum=None):
    """Root-mean-square norm of residual + dropout(x).  out_type torch.int8 gives 8-bit rows and their scales.  The sum is
    kept (unless keep_sum is false) where it is another than x.  out, scale and sum may be passed; sum may be residual."""
    kind = _kind(x, _TYPES, "x")
    rows, cols = x.shape if x.dim() == 2 else _refuse("x: a 2-D tensor")
    device = x.device
    at, stride = _rows("x", x)
    res_at, res_stride = (None, 0) if residual is None else _rows("residual", residual, x)
    gain_at = _array("gain", gain, cols, torch.float32, x)
    if out is None:
        out = torch.empty((rows, cols), dtype=out_type or x.dtype, device=device)
    if out_type is not None and out.dtype is not out_type:
        _refuse("out is not of out_type")
    bytes_out = out.dtype is torch.int8
    out_at, out_stride = _rows("out", out, x, out.dtype if bytes_out else None)
    scale_at = None
    if bytes_out:
        if scale is None:
            scale = torch.empty(rows, dtype=torch.float32, device=device)
        scale_at = _array("scale", scale, rows, torch.float32, x)
    elif scale is not None:
        _refuse("scale belongs to an 8-bit out")
    if sum is None and keep_sum and (residual is not None or drop != 0.0):
        sum = torch.empty((rows, cols), dtype=x.dtype, device=device)
    sum_at, sum_stride = (None, 0) if sum is None else _rows("sum", sum, x)
    rstd = torch.empty(rows, dtype=torch.float32, device=device) if keep_rstd else None
    _call(load().gv_norm_rows, device, rows, cols, kind, at, stride, res_at, res_stride, gain_at, eps, drop, seed, first_row,
          sum_at, sum_stride, GV_I8 if bytes_out else kind, out_at, out_stride, scale_at, rstd.data_ptr() if keep_rstd else None)
    return NormRows(out, scale, sum, rstd)


@functools.lru_cache(maxsize=256)
def gv_norm_rows_workspace(rows, cols):
    """Bytes of scratch that the gradient of the gain takes."""
    n = C.c_uint64()
    rc = load().gv_norm_rows_workspace(rows, cols, C.byref(n))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())
    return n.value


def gv_norm_rows_backward(grad_out, sum, gain, rstd, *, grad_sum=None, drop=0.0, seed=0, first_row=0, keep_residual=None,
                          keep_gain=True):
    """Gradients of gv_norm_rows for x, residual and gain.  The residual's is made where keep_residual asks for it (by
    default: where grad_sum is passed); without dropout it is x's, the same tensor."""
    kind = _kind(grad_out, _TYPES, "grad_out")
    rows, cols = grad_out.shape if grad_out.dim() == 2 else _refuse("grad_out: a 2-D tensor")
    device = grad_out.device
    go_at, go_stride = _rows("grad_out", grad_out)
    sum_at, sum_stride = _rows("sum", sum, grad_out)
    gs_at, gs_stride = (None, 0) if grad_sum is None else _rows("grad_sum", grad_sum, grad_out)
    gain_at = _array("gain", gain, cols, torch.float32, grad_out)
    rstd_at = _array("rstd", rstd, rows, torch.float32, grad_out)
    grad_x = torch.empty((rows, cols), dtype=grad_out.dtype, device=device)
    grad_residual = None
    if grad_sum is not None if keep_residual is None else keep_residual:
        grad_residual = grad_x if drop == 0.0 else torch.empty_like(grad_x)
    apart = grad_residual is not None and grad_residual is not grad_x
    grad_gain, space, size = None, None, 0
    if keep_gain:
        grad_gain = torch.empty(cols, dtype=torch.float32, device=device)
        size = gv_norm_rows_workspace(rows, cols)
        space = torch.empty(size, dtype=torch.uint8, device=device)
    _call(load().gv_norm_rows_backward, device, rows, cols, kind, go_at, go_stride, sum_at, sum_stride, gain_at, rstd_at, gs_at,
          gs_stride, drop, seed, first_row, grad_x.data_ptr(), cols, grad_residual.data_ptr() if apart else None, cols,
          grad_gain.data_ptr() if keep_gain else None, space.data_ptr() if keep_gain else None, size)
    return NormGrads(grad_x, grad_residual, grad_gain)


def gv_quantize_rows(x, *, group=32):
    """(codes uint8[rows][16 ceil(cols / 32)], scales bfloat16[rows][ceil(cols / group)]): the table of x in 4 bits."""
    kind = _kind(x, _TYPES, "x")
    rows, cols = x.shape if x.dim() == 2 else _refuse("x: a 2-D tensor")
    at, stride = _rows("x", x)
    codes = torch.empty((rows, 16 * (-(-cols // 32))), dtype=torch.uint8, device=x.device)
    scales = torch.empty((rows, -(-cols // group) if group > 0 else 0), dtype=torch.bfloat16, device=x.device)
    _call(load().gv_quantize_rows, x.device, rows, cols, kind, at, stride, group, codes.data_ptr(), scales.data_ptr())
    return codes, scales


def gv_score_rows(codes, scales, x, *, group=32, scale=None, out=None):
    """float32[queries][rows]: the scores of the query rows x (8-bit rows with their `scale`) against every row of the
    table that gv_quantize_rows made."""
    kind = _kind(x, _TYPES_AND_BYTES, "x")
    queries, cols = x.shape if x.dim() == 2 else _refuse("x: a 2-D tensor")
    rows = codes.shape[0]
    at, stride = _rows("x", x)
    codes_at = _array("codes", codes, rows * 16 * (-(-cols // 32)), torch.uint8, x)
    scales_at = _array("scales", scales, rows * (-(-cols // group)) if group > 0 else 0, torch.bfloat16, x)
    if out is None:
        out = torch.empty((queries, rows), dtype=torch.float32, device=x.device)
    elif out.shape != (queries, rows) or out.dtype is not torch.float32 or out.device != x.device:
        _refuse("out: float32[queries][rows]")
    out_at, out_stride = _rows("out", out)
    scale_at = None if scale is None else _array("scale", scale, queries, torch.float32, x)
    _call(load().gv_score_rows, x.device, rows, cols, group, codes_at, scales_at, queries, kind, at, stride, scale_at, out_at,
          out_stride)
    return out
