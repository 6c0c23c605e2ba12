"""The operators on rows in device memory (include/gvhot.h) for tensors of torch: shapes, strides and types are read
from the tensors, results that the caller does not pass are allocated, and the kernels go to torch's current stream
of the tensors' GPU.  Rows are 2-D tensors whose last dimension is contiguous; their rows may lie further apart.
No arithmetic happens here.

The calls record no graph for autograd: gradients are calls of their own (gv_norm_rows_backward; dropout's is dropout).  So
where gradients are enabled and a tensor of a floating result asks for one, a call refuses: it belongs under torch.no_grad(), or
takes detached tensors.  Codes, of 8-bit rows and of tables, are constants.
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


def _without_graph(*tensors):
    if any(t is not None and t.requires_grad for t in tensors):
        _refuse("no graph is recorded here, and a tensor asks for gradients: call under torch.no_grad() or pass it detached "
                "(gradients are calls of their own: gv_norm_rows_backward, gv_drop_rows)")


# A call that finds its kernel's launch waiting for nothing is as long as the host takes for it, 3.5 us of which are the launch:
# so torch is asked in the ways that take it least.  The current stream of a GPU as an address, and the current GPU:
# the public ways make a Stream object and look whether torch is initialised first (1.9 and 0.25 us instead of 0.1 each).
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda gpu: torch.cuda.current_stream(gpu).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_recording = torch.is_grad_enabled
# a passed tensor that was written to: autograd raises where it had kept what was there
_written = torch.autograd.graph.increment_version
_f32, _int8, _uint8, _bf16 = torch.float32, torch.int8, torch.uint8, torch.bfloat16


def _first(name, t, kinds=_TYPES):
    """(address, stride, rows, cols, type, GPU) of the matrix of rows that the others of a call have to be like."""
    kind = kinds.get(t.dtype)
    if kind is None or not t.is_cuda:
        _refuse(f"{name}: rows of {', '.join(map(str, kinds))} in device memory are asked for")
    shape = t.shape
    if len(shape) != 2:
        _refuse(f"{name}: a 2-D tensor")
    rows, cols = shape
    stride, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(f"{name}: the values of a row lie together")
    return t.data_ptr(), (stride if rows > 1 else cols), rows, cols, kind, t.get_device()


def _rows(name, t, rows, cols, dtype, gpu):
    """(address, stride) of another matrix of rows."""
    if t.shape != (rows, cols) or t.dtype is not dtype or t.get_device() != gpu:
        _refuse(f"{name}: {rows} rows of {cols} {dtype} on the same GPU are asked for")
    stride, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(f"{name}: the values of a row lie together")
    return t.data_ptr(), (stride if rows > 1 else cols)


def _array(name, t, size, dtype, gpu):
    """Address of a contiguous array of `size` values."""
    if t.dtype is not dtype or t.numel() != size or not t.is_contiguous() or t.get_device() != gpu:
        _refuse(f"{name}: {size} contiguous values of {dtype} on the same GPU are asked for")
    return t.data_ptr()


def _call(entry, gpu, *args):
    if gpu == _current_device():
        rc = entry(*args, _stream_of(gpu))
    else:
        with torch.cuda.device(gpu):
            rc = entry(*args, _stream_of(gpu))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())


def _like(x, rows, cols):
    """A new matrix of x's shape and type (the call that reads them from x takes two thirds of the other's time)."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty((rows, cols))


def gv_drop_rows(x, drop, seed, *, first_row=0, out=None):
    """Dropout of rows.  The gradient of x is the same call, with the same drop, seed and first_row, on out's gradient."""
    at, stride, rows, cols, kind, gpu = _first("x", x)
    passed = out is not None
    if _recording() and (x.requires_grad or passed):
        _without_graph(x, out)
    if passed:
        out_at, out_stride = _rows("out", out, rows, cols, x.dtype, gpu)
    else:
        out = _like(x, rows, cols)
        out_at, out_stride = out.data_ptr(), cols
    _call(load().gv_drop_rows, gpu, rows, cols, kind, at, stride, drop, seed, first_row, out_at, out_stride)
    if passed:
        _written(out)
    return out


def gv_norm_rows(x, gain, residual=None, *, eps=1e-6, drop=0.0, seed=0, first_row=0, out_type=None, keep_sum=True,
                 keep_rstd=False, out=None, scale=None, sum=None):
    """Root-mean-square norm of residual + dropout(x).  out_type torch.int8 gives 8-bit rows and their scales.  The sum is
    kept (unless keep_sum is false) where it is another than x.  out, scale and sum may be passed; sum may be residual."""
    at, stride, rows, cols, kind, gpu = _first("x", x)
    dtype = x.dtype
    gain_at = _array("gain", gain, cols, _f32, gpu)
    res_at, res_stride = (None, 0) if residual is None else _rows("residual", residual, rows, cols, dtype, gpu)
    passed = (out, scale, sum) if out is not None or scale is not None or sum is not None else ()
    if out is None:
        out_type = out_type or dtype
        out = _like(x, rows, cols) if out_type is dtype else x.new_empty((rows, cols), dtype=out_type)
        out_at, out_stride = out.data_ptr(), cols
    else:
        out_type = out_type or out.dtype
        out_at, out_stride = _rows("out", out, rows, cols, out_type, gpu)
    if out_type is not dtype and out_type is not _int8:
        _refuse("out: the type of x, or torch.int8")
    scale_at = sum_at = rstd = rstd_at = None
    sum_stride, out_kind = 0, kind
    if out_type is _int8:
        out_kind = GV_I8
        if scale is None:
            scale = gain.new_empty(rows)
            scale_at = scale.data_ptr()
        else:
            scale_at = _array("scale", scale, rows, _f32, gpu)
    elif scale is not None:
        _refuse("scale belongs to an 8-bit out")
    if sum is not None:
        sum_at, sum_stride = _rows("sum", sum, rows, cols, dtype, gpu)
    elif keep_sum and (residual is not None or drop != 0.0):
        sum = _like(x, rows, cols)
        sum_at, sum_stride = sum.data_ptr(), cols
    if keep_rstd:
        rstd = gain.new_empty(rows)
        rstd_at = rstd.data_ptr()
    if _recording() and (passed or x.requires_grad or gain.requires_grad or (residual is not None and residual.requires_grad)):
        _without_graph(*passed)
        if out_type is not _int8:
            _without_graph(x, residual, gain)
        elif sum is not None:
            _without_graph(x, residual)
    _call(load().gv_norm_rows, gpu, rows, cols, kind, at, stride, res_at, res_stride, gain_at, eps, drop, seed, first_row,
          sum_at, sum_stride, out_kind, out_at, out_stride, scale_at, rstd_at)
    if passed:
        _written([t for t in passed if t is not None])
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
    go_at, go_stride, rows, cols, kind, gpu = _first("grad_out", grad_out)
    dtype = grad_out.dtype
    sum_at, sum_stride = _rows("sum", sum, rows, cols, dtype, gpu)
    gs_at, gs_stride = (None, 0) if grad_sum is None else _rows("grad_sum", grad_sum, rows, cols, dtype, gpu)
    gain_at = _array("gain", gain, cols, _f32, gpu)
    rstd_at = _array("rstd", rstd, rows, _f32, gpu)
    if _recording() and (grad_out.requires_grad or sum.requires_grad or gain.requires_grad or rstd.requires_grad
                         or (grad_sum is not None and grad_sum.requires_grad)):
        _without_graph(grad_out, sum, gain, rstd, grad_sum)
    grad_x = _like(grad_out, rows, cols)
    grad_residual = res_at = grad_gain = gain_to = space_at = None
    size = 0
    if grad_sum is not None if keep_residual is None else keep_residual:
        if drop == 0.0:
            grad_residual = grad_x
        else:
            grad_residual = _like(grad_out, rows, cols)
            res_at = grad_residual.data_ptr()
    if keep_gain:
        size = gv_norm_rows_workspace(rows, cols)
        grad_gain = torch.empty_like(gain)
        gain_to = grad_gain.data_ptr()
        if size:
            space = gain.new_empty(size // 4)
            space_at = space.data_ptr()
    _call(load().gv_norm_rows_backward, gpu, rows, cols, kind, go_at, go_stride, sum_at, sum_stride, gain_at, rstd_at, gs_at,
          gs_stride, drop, seed, first_row, grad_x.data_ptr(), cols, res_at, cols, gain_to, space_at, size)
    return NormGrads(grad_x, grad_residual, grad_gain)


def _parts(cols, size):
    return -(-cols // size) if size > 0 else 0


def gv_quantize_rows(x, *, group=32):
    """(codes uint8[rows][16 ceil(cols / 32)], scales bfloat16[rows][ceil(cols / group)]): the table of x in 4 bits."""
    at, stride, rows, cols, kind, gpu = _first("x", x)
    codes = torch.empty((rows, 16 * _parts(cols, 32)), dtype=_uint8, device=x.device)
    scales = torch.empty((rows, _parts(cols, group)), dtype=_bf16, device=x.device)
    _call(load().gv_quantize_rows, gpu, rows, cols, kind, at, stride, group, codes.data_ptr(), scales.data_ptr())
    return codes, scales


def gv_score_rows(codes, scales, x, *, group=32, scale=None, out=None):
    """float32[queries][rows]: the scores of the query rows x (8-bit rows with their `scale`) against every row of the
    table that gv_quantize_rows made."""
    at, stride, queries, cols, kind, gpu = _first("x", x, _TYPES_AND_BYTES)
    rows = codes.shape[0]
    codes_at = _array("codes", codes, rows * 16 * _parts(cols, 32), _uint8, gpu)
    scales_at = _array("scales", scales, rows * _parts(cols, group), _bf16, gpu)
    passed = out is not None
    if passed:
        out_at, out_stride = _rows("out", out, queries, rows, _f32, gpu)
    else:
        out = (x if scale is None else scale).new_empty((queries, rows), dtype=_f32)
        out_at, out_stride = out.data_ptr(), rows
    scale_at = None if scale is None else _array("scale", scale, queries, _f32, gpu)
    if _recording() and (passed or x.requires_grad or scales.requires_grad or (scale is not None and scale.requires_grad)):
        _without_graph(x, scales, scale, out)
    _call(load().gv_score_rows, gpu, rows, cols, group, codes_at, scales_at, queries, kind, at, stride, scale_at, out_at,
          out_stride)
    if passed:
        _written(out)
    return out
