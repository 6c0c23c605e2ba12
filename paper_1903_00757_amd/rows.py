"""The operators on rows in device memory (include/gvhot.h) for tensors of torch: shapes, strides and types are read
from the tensors, results that the caller does not pass are allocated, and the kernels go to torch's current stream
of the tensors' GPU.  Rows are 2-D tensors whose last dimension is contiguous; their rows may lie further apart.
No arithmetic happens here.

The calls record no graph for autograd: gradients are calls of their own (gv_norm_rows_backward, gv_lookup_rows_backward,
gv_dense_rows_backward; dropout's is dropout).  So where gradients are enabled and a tensor of a floating result asks for one, a
call refuses: it belongs under torch.no_grad(), or takes detached tensors.  Codes, of 8-bit rows and of tables, are constants.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import NamedTuple, Optional

import torch

from .binding import GV_ACT_NONE, GV_BF16, GV_F16, GV_F32, GV_I8, GV_I32, GV_I64, GV_OK, GvError, load

__all__ = ["NormRows", "NormGrads", "gv_drop_rows", "gv_norm_rows", "gv_norm_rows_workspace", "gv_norm_rows_backward",
           "gv_quantize_rows", "gv_score_rows", "gv_lookup_rows", "gv_lookup_rows_workspace", "gv_lookup_rows_backward",
           "DenseRows", "DenseGrads", "gv_dense_rows", "gv_dense_rows_workspace", "gv_dense_rows_backward", "gv_dense_rows_backward_workspace",
           "Selection", "gv_select_rows", "gv_select_rows_workspace"]

_TYPES = {torch.float32: GV_F32, torch.bfloat16: GV_BF16, torch.float16: GV_F16}
_TYPES_AND_BYTES = dict(_TYPES)
_TYPES_AND_BYTES[torch.int8] = GV_I8
_TYPES_AND_WHOLE = dict(_TYPES_AND_BYTES)
_TYPES_AND_WHOLE.update({torch.uint8: GV_I8, torch.bool: GV_I8, torch.int32: GV_I32, torch.int64: GV_I64})
_INDICES = {torch.int32: GV_I32, torch.int64: GV_I64}


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


class DenseRows(NamedTuple):
    out: torch.Tensor
    pre: Optional[torch.Tensor]


class DenseGrads(NamedTuple):
    """Of a layer; None where it was not asked for.  The residual's is the gradient that came in."""
    x: Optional[torch.Tensor]
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]


class Selection(NamedTuple):
    """What gv_select_rows gives, [groups][best]; -1 and -inf where there was nothing more to select."""
    parent: torch.Tensor  # int64: the beam, counted over all queries
    row: torch.Tensor     # int64
    total: torch.Tensor   # float32


def _refuse(text):
    raise ValueError(text)


def _without_graph(*tensors):
    if any(t is not None and t.requires_grad for t in tensors):
        _refuse("no graph is recorded here, and a tensor asks for gradients: call under torch.no_grad() or pass it detached "
                "(gradients are calls of their own: gv_norm_rows_backward, gv_drop_rows, gv_lookup_rows_backward, gv_dense_rows_backward)")


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


def _index(t, gpu):
    """(address, stride, count, type) of the indices of a batch."""
    kind = _INDICES.get(t.dtype)
    if kind is None or t.get_device() != gpu:
        _refuse("index: int32 or int64 on the same GPU are asked for")
    if t.dim() != 1:
        _refuse("index: a 1-D tensor")
    return t.data_ptr(), t.stride(0), t.numel(), kind


def gv_lookup_rows(table, index, *, scale=1.0, out_type=None, out=None):
    """Rows of the table by index (a 1-D tensor, a column of pairs for instance), times scale; zeros where an index names no
    row.  Types of whole numbers are copied.  The gradient of the table is gv_lookup_rows_backward."""
    at, stride, rows, cols, kind, gpu = _first("table", table, _TYPES_AND_WHOLE)
    index_at, index_stride, count, index_kind = _index(index, gpu)
    passed = out is not None
    dtype = out_type or (out.dtype if passed else table.dtype)
    out_kind = kind if dtype is table.dtype else _TYPES.get(dtype)
    if out_kind is None or (out_kind != kind and kind > GV_F16):
        _refuse("out: float32, bfloat16 or float16, or the table's type")
    if passed:
        out_at, out_stride = _rows("out", out, count, cols, dtype, gpu)
    else:
        out = table.new_empty((count, cols), dtype=dtype)
        out_at, out_stride = out.data_ptr(), cols
    if _recording() and (table.requires_grad or passed):
        _without_graph(table, out)
    _call(load().gv_lookup_rows, gpu, count, index_at, index_stride, index_kind, rows, cols, kind, at, stride, scale, out_kind, out_at,
          out_stride)
    if passed:
        _written(out)
    return out


@functools.lru_cache(maxsize=256)
def gv_lookup_rows_workspace(count, rows, cols, add=False):
    """Bytes of scratch that the gradient of a batch of `count` rows takes."""
    n = C.c_uint64()
    rc = load().gv_lookup_rows_workspace(count, rows, cols, 1 if add else 0, C.byref(n))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())
    return n.value


def gv_lookup_rows_backward(grad_out, index, rows, *, scale=1.0, out_type=None, out=None, add=False):
    """The gradient of a table of `rows` rows: the rows of grad_out added up by index, times scale.  With add, out's rows that the
    batch names get theirs added and the others stay: gv_lookup_rows_backward(g, index, n, scale=-rate, out=table, add=True) is a
    step on the table."""
    at, stride, count, cols, kind, gpu = _first("grad_out", grad_out)
    index_at, index_stride, named, index_kind = _index(index, gpu)
    if named != count:
        _refuse(f"index: {count} of them are asked for")
    passed = out is not None
    if add and not passed:
        _refuse("add: out is asked for")
    dtype = out_type or (out.dtype if passed else grad_out.dtype)
    out_kind = _TYPES.get(dtype)
    if out_kind is None:
        _refuse("out: float32, bfloat16 or float16")
    if passed:
        out_at, out_stride = _rows("out", out, rows, cols, dtype, gpu)
    else:
        out = grad_out.new_empty((rows, cols), dtype=dtype)
        out_at, out_stride = out.data_ptr(), cols
    if _recording() and (grad_out.requires_grad or passed):
        _without_graph(grad_out, out)
    add = bool(add)
    size = gv_lookup_rows_workspace(count, rows, cols, add)
    space = torch.empty(size, dtype=_uint8, device=grad_out.device) if size else None
    _call(load().gv_lookup_rows_backward, gpu, count, index_at, index_stride, index_kind, rows, cols, kind, at, stride, scale, add, out_kind,
          out_at, out_stride, space.data_ptr() if size else None, size)
    if passed:
        _written(out)
    return out


@functools.lru_cache(maxsize=256)
def gv_dense_rows_workspace(rows, cols, outs, type):
    """Bytes of scratch that a layer takes."""
    n = C.c_uint64()
    rc = load().gv_dense_rows_workspace(rows, cols, outs, type, C.byref(n))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())
    return n.value


def gv_dense_rows(x, weight, bias=None, residual=None, *, act=GV_ACT_NONE, keep_pre=False, out=None):
    """residual + act(x weight^T + bias).  weight is [outs][cols], all are of x's type.  keep_pre keeps what the activation is taken
    of, for gv_dense_rows_backward.  out may be passed, and may be residual."""
    at, stride, rows, cols, kind, gpu = _first("x", x)
    dtype = x.dtype
    if weight.dim() != 2:
        _refuse("weight: a 2-D tensor")
    outs = weight.shape[0]
    weight_at, weight_stride = _rows("weight", weight, outs, cols, dtype, gpu)
    bias_at = None if bias is None else _array("bias", bias, outs, dtype, gpu)
    res_at, res_stride = (None, 0) if residual is None else _rows("residual", residual, rows, outs, dtype, gpu)
    passed = out is not None
    if passed:
        out_at, out_stride = _rows("out", out, rows, outs, dtype, gpu)
    else:
        out = x.new_empty((rows, outs))
        out_at, out_stride = out.data_ptr(), outs
    if _recording() and (passed or x.requires_grad or weight.requires_grad or bias is not None or residual is not None):
        _without_graph(x, weight, bias, residual, out)
    pre = x.new_empty((rows, outs)) if keep_pre else None
    size = gv_dense_rows_workspace(rows, cols, outs, kind)
    space = torch.empty(size, dtype=_uint8, device=x.device) if size else None
    _call(load().gv_dense_rows, gpu, rows, cols, outs, kind, at, stride, weight_at, weight_stride, bias_at, act, res_at, res_stride,
          pre.data_ptr() if keep_pre else None, outs, out_at, out_stride, space.data_ptr() if size else None, size)
    if passed:
        _written(out)
    return DenseRows(out, pre)


@functools.lru_cache(maxsize=256)
def gv_dense_rows_backward_workspace(rows, cols, outs, type, act, keep_x=True, keep_weight=True, keep_bias=False):
    """Bytes of scratch that the gradients of a layer take."""
    n = C.c_uint64()
    rc = load().gv_dense_rows_backward_workspace(rows, cols, outs, type, act, keep_x, keep_weight, keep_bias, C.byref(n))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())
    return n.value


def gv_dense_rows_backward(grad_out, x, weight, pre=None, *, act=GV_ACT_NONE, keep_x=True, keep_weight=True, keep_bias=False):
    """Gradients of gv_dense_rows for x, weight and bias; the residual's is grad_out.  pre is what the layer kept, where it has an
    activation."""
    at, stride, rows, outs, kind, gpu = _first("grad_out", grad_out)
    dtype = grad_out.dtype
    if x.dim() != 2:
        _refuse("x: a 2-D tensor")
    cols = x.shape[1]
    x_at, x_stride = _rows("x", x, rows, cols, dtype, gpu)
    weight_at, weight_stride = _rows("weight", weight, outs, cols, dtype, gpu)
    pre_at, pre_stride = (None, 0) if pre is None else _rows("pre", pre, rows, outs, dtype, gpu)
    if pre is None and act != GV_ACT_NONE:
        _refuse("pre: an activation's gradient is taken of it")
    if _recording() and (grad_out.requires_grad or x.requires_grad or weight.requires_grad or pre is not None):
        _without_graph(grad_out, x, weight, pre)
    keep_x, keep_weight, keep_bias = bool(keep_x), bool(keep_weight), bool(keep_bias)
    grad_x = grad_out.new_empty((rows, cols)) if keep_x else None
    grad_weight = grad_out.new_empty((outs, cols)) if keep_weight else None
    grad_bias = grad_out.new_empty(outs) if keep_bias else None
    size = gv_dense_rows_backward_workspace(rows, cols, outs, kind, act, keep_x, keep_weight, keep_bias)
    space = torch.empty(size, dtype=_uint8, device=grad_out.device) if size else None
    _call(load().gv_dense_rows_backward, gpu, rows, cols, outs, kind, at, stride, x_at, x_stride, weight_at, weight_stride, act, pre_at,
          pre_stride, grad_x.data_ptr() if keep_x else None, cols, grad_weight.data_ptr() if keep_weight else None, cols,
          grad_bias.data_ptr() if keep_bias else None, space.data_ptr() if size else None, size)
    return DenseGrads(grad_x, grad_weight, grad_bias)


@functools.lru_cache(maxsize=256)
def gv_select_rows_workspace(queries, rows, beams, best):
    """Bytes of scratch that a selection takes."""
    n = C.c_uint64()
    rc = load().gv_select_rows_workspace(queries, rows, beams, best, C.byref(n))
    if rc != GV_OK:
        raise GvError(rc, load().gv_last_error(None).decode())
    return n.value


def gv_select_rows(scores, best, *, beams=1, totals=None, done=None, end=0, log_softmax=True):
    """The best rows over the scores of each group of `beams` queries: by totals + log softmax of the scores, or totals + scores.
    done (bool): beams that have ended offer row `end` alone.  gv_lookup_rows(states, got.parent.view(-1)) gives the states that
    belong to what was selected."""
    kind = _TYPES.get(scores.dtype)
    if kind is None or not scores.is_cuda:
        _refuse(f"scores: {', '.join(map(str, _TYPES))} in device memory are asked for")
    if scores.dim() != 2:
        _refuse("scores: a 2-D tensor")
    queries, rows = scores.shape
    stride, step = scores.stride()
    if step != 1 and rows > 1:
        _refuse("scores: the scores of a query lie together")
    gpu = scores.get_device()
    totals_at = None if totals is None else _array("totals", totals, queries, _f32, gpu)
    done_at = None if done is None else _array("done", done, queries, torch.bool, gpu)
    if _recording() and (scores.requires_grad or (totals is not None and totals.requires_grad)):
        _without_graph(scores, totals)
    size = gv_select_rows_workspace(queries, rows, beams, best)
    groups = queries // beams
    at = torch.empty((2, groups, best), dtype=torch.int64, device=scores.device)
    parent, row = at[0], at[1]
    total = torch.empty((groups, best), dtype=_f32, device=scores.device)
    space = torch.empty(size, dtype=_uint8, device=scores.device) if size else None
    first = at.data_ptr()
    _call(load().gv_select_rows, gpu, queries, rows, kind, scores.data_ptr(), stride if queries > 1 else rows, beams, totals_at, done_at, end,
          bool(log_softmax), best, first, first + 8 * groups * best, total.data_ptr(), space.data_ptr() if size else None, size)
    return Selection(parent, row, total)
