"""Binding of include/liec_train.h: the operators around the backward pass whose gradients a compressed step takes.

Tensors of N workers carry the workers as their leading dimension.  Every function enqueues its kernels on torch's
current stream of the tensors' device and returns; scratch comes from torch's allocator.  Only arguments are checked and
marshalled here.
"""
from __future__ import annotations

import ctypes
import math
from array import array
from itertools import repeat
from operator import attrgetter, floordiv
from typing import Optional, Sequence, Tuple

import torch

from .binding import _check, lib

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_dtype_code = _DTYPES.get
_dtype_of = attrgetter("dtype")
_Tensor = torch.Tensor


def _stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


# the same without an object for the stream (1 us of a call), where torch has it
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)


def _call(name: str, device: int, *args) -> None:
    """The entry point `name` on the current stream of `device`, which is the current device while it launches."""
    function = getattr(lib(), name)
    if torch.cuda.current_device() == device:
        status = function(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = function(*args, _stream(device))
    if status:
        _check(status, name)


# ---- gradients ------------------------------------------------------------------------------------------------------
def _grad_table(grads: Sequence[torch.Tensor], N: int, whole: bool, device: int) -> Tuple[array, int]:
    """(liec_grad_tensor of each tensor, as the words the struct is made of; values of a worker in all)"""
    types = set(map(_dtype_of, grads))
    if not types <= _DTYPES.keys() or not set(map(_Tensor.get_device, grads)) <= {device}:
        raise TypeError("gradients must be float32, bfloat16 or float16 tensors on one GPU")
    counts = list(map(_Tensor.numel, grads))
    contiguous = all(map(_Tensor.is_contiguous, grads))
    strides = counts
    if whole:
        if not contiguous:
            raise ValueError("gradients of one worker must be contiguous")
    else:
        try:
            leading = set(map(_Tensor.size, grads, repeat(0)))
        except IndexError:                                     # a tensor without dimensions
            leading = {None}
        if not leading <= {N}:
            raise ValueError(f"every gradient needs {N} workers as its leading dimension: {[tuple(t.shape) for t in grads][:8]}")
        counts = strides = list(map(floordiv, counts, repeat(N)))
        if not contiguous:
            if not all(t[0].is_contiguous() for t in grads):
                raise ValueError("the gradients of a worker must be contiguous within each tensor")
            strides = [n if t.is_contiguous() else t.stride(0) for t, n in zip(grads, counts)]
    table = array("q", bytes(32 * len(counts)))
    table[0::4] = array("q", map(_Tensor.data_ptr, grads))
    table[1::4] = array("q", counts)
    table[2::4] = array("q", strides)
    if types != {torch.float32}:                               # whose code is 0
        table[3::4] = array("q", map(_dtype_code, map(_dtype_of, grads)))
    return table, sum(counts)


def _grad_args(grads, norms, workers):
    """(tensors' table, values of a worker, N, device, workspace, its bytes)"""
    if norms is None and not grads:
        raise ValueError("no gradients, and no norms to tell the number of workers")
    first = grads[0] if grads else norms
    device = first.get_device()
    if device < 0:
        raise TypeError("gradients must be on the GPU")
    if workers is not None and workers != 1:
        raise ValueError("workers is 1 for tensors of one worker, or None for tensors with a leading dimension of workers")
    N = 1 if workers else norms.numel() if norms is not None else first.shape[0] if first.dim() else 0
    if norms is not None:
        if norms.dtype != torch.float32 or norms.get_device() != device or norms.dim() != 1 or not norms.is_contiguous():
            raise TypeError("norms must be a contiguous float32 vector on the gradients' GPU")
        if norms.numel() != N:
            raise ValueError(f"norms has {norms.numel()} values, expected {N}")
    if N < 1:
        raise ValueError("no workers")
    table, total = _grad_table(grads, N, workers == 1, device)
    need = lib().liec_grads_workspace(N, len(grads))
    if need < 0:
        raise ValueError(f"{len(grads)} tensors of {N} workers are more than the library takes")
    return table, total, N, device, torch.empty(need, dtype=torch.uint8, device=first.device), need


def _optional(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def liec_grad_norm(grads: Sequence[torch.Tensor], norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> torch.Tensor:
    """Global l2 norm of each worker's gradients over all tensors, [N] float32, summed in 64 bits.  `workers=1`: the
    tensors, of any shape, belong to one worker; otherwise their leading dimension is the workers'."""
    table, _, N, device, ws, need = _grad_args(grads, norms, workers)
    if norms is None:
        norms = torch.empty(N, dtype=torch.float32, device=ws.device)
    _call("liec_grad_norm", device, table.buffer_info()[0], len(grads), N, norms.data_ptr(), ws.data_ptr(), need)
    return norms


def liec_clip_grads(grads: Sequence[torch.Tensor], max_norm: float, norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> None:
    """Scales each worker's gradients in place so that their global norm is at most max_norm; `norms`, when given,
    receives the norms before that."""
    table, _, N, device, ws, need = _grad_args(grads, norms, workers)
    _call("liec_clip_grads", device, table.buffer_info()[0], len(grads), N, max_norm, _optional(norms), ws.data_ptr(), need)


def liec_gather_grads(grads: Sequence[torch.Tensor], rows: torch.Tensor, max_norm: float = math.inf, norms: Optional[torch.Tensor] = None,
                      workers: Optional[int] = None) -> None:
    """Puts each worker's tensors one after the other into its row of `rows` ([N, d] float32, as LiecContext.step reads
    it), scaled so that the row's norm is at most max_norm."""
    table, total, N, device, ws, need = _grad_args(grads, norms, workers)
    if rows.dtype != torch.float32 or rows.get_device() != device or rows.dim() != 2 or (rows.stride(1) != 1 and rows.shape[1] > 1):
        raise TypeError("rows must be a float32 [N, d] tensor on the gradients' GPU whose rows are contiguous")
    if rows.shape[0] != N or rows.shape[1] != total:
        raise ValueError(f"rows has shape {tuple(rows.shape)}, expected {(N, total)}")
    _call("liec_gather_grads", device, table.buffer_info()[0], len(grads), N, rows.data_ptr(), rows.stride(0), max_norm, _optional(norms), ws.data_ptr(), need)


# ---- layer normalisation --------------------------------------------------------------------------------------------
class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


_ref = ctypes.byref


class _Param(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


def _workers_of(x: torch.Tensor, params) -> Tuple[int, int, int]:
    """(N, R, C) of activations x under these weights, biases and their gradients (some of them None)."""
    shape = x.shape
    C = shape[-1] if shape else 0
    if C < 1:
        raise ValueError(f"activations of shape {tuple(shape)} have no columns")
    N = 0
    for p in params:
        if p is None:
            continue
        dims = p.dim()
        if dims not in (1, 2) or p.size(-1) != C or (p.stride(-1) != 1 and C > 1):
            raise ValueError(f"a weight or bias of shape {tuple(p.shape)} does not fit {C} columns, or its columns are not contiguous")
        if dims == 2:
            N = p.size(0)
            if len(shape) < 2 or N != shape[0] or not N:
                raise ValueError(f"weights of {N} workers do not fit activations of shape {tuple(shape)}")
    if N:
        return N, x.numel() // (N * C), C
    if len(shape) == 3 and shape[0] and not x.is_contiguous():
        return shape[0], shape[1], C
    return 1, x.numel() // C, C


def _rows(t: torch.Tensor, N: int, R: int, C: int, what: str):
    """liec_rows of a tensor that is N workers' R rows of C columns."""
    if t.is_contiguous():
        return _ref(_Rows(t.data_ptr(), R * C, C))
    try:
        v = t.view(N, R, C)
    except RuntimeError:
        raise ValueError(f"{what} of strides {t.stride()} is not {N} workers' rows at equal distances") from None
    if C > 1 and v.stride(2) != 1:
        raise ValueError(f"the columns of {what} must be contiguous")
    return _ref(_Rows(t.data_ptr(), v.stride(0), v.stride(1)))


def _like(t: torch.Tensor, x: torch.Tensor, what: str) -> None:
    if t.dtype != x.dtype or t.get_device() != x.get_device():
        raise TypeError(f"{what} must have the activations' type and device")
    if t.shape != x.shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(x.shape)}")


def _param(p: Optional[torch.Tensor], dtype, device: int):
    if p is None:
        return None
    if p.dtype != dtype or p.get_device() != device:
        raise TypeError("weights, biases and their gradients must be of one type, float32, bfloat16 or float16, on the activations' GPU")
    return _ref(_Param(p.data_ptr(), p.stride(0) if p.dim() == 2 else 0))


def _param_type(*params):
    """(type, its code) of the first one that is there."""
    for p in params:
        if p is not None:
            code = _dtype_code(p.dtype)
            if code is None:
                raise TypeError("weights, biases and their gradients must be float32, bfloat16 or float16")
            return p.dtype, code
    return None, 0


def liec_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Layer normalisation over the last dimension: (y, mean, rstd), the latter two float32 of x's other dimensions.
    weight and bias: [C], or [N, C] for the N workers of x's leading dimension (columns of a models tensor, say).
    `out` may be x."""
    code, device = _dtype_code(x.dtype), x.get_device()
    if code is None or device < 0:
        raise TypeError("activations must be float32, bfloat16 or float16 on the GPU")
    N, R, C = _workers_of(x, (weight, bias))
    ptype, pcode = _param_type(weight, bias)
    w, b = _param(weight, ptype, device), _param(bias, ptype, device)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _like(out, x, "out")
    lead = x.shape[:-1]
    mean = torch.empty(lead, dtype=torch.float32, device=x.device)
    rstd = torch.empty(lead, dtype=torch.float32, device=x.device)
    _call("liec_layer_norm", device, _rows(x, N, R, C, "x"), w, b, _rows(out, N, R, C, "out"), mean.data_ptr(), rstd.data_ptr(), N, R, C, eps, code, pcode)
    return out, mean, rstd


def liec_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                             dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             need_dx: bool = True) -> Optional[torch.Tensor]:
    """Gradients of liec_layer_norm: returns dx (a new tensor unless one is given, which may be dy or x; None with
    need_dx=False) and writes the gradients of weight and bias into dweight and dbias where they are given: [N, C] takes
    each worker's own sum (columns of the gradient rows of a step, say), [C] the sum over everything."""
    code, device = _dtype_code(x.dtype), x.get_device()
    if code is None or device < 0:
        raise TypeError("activations must be float32, bfloat16 or float16 on the GPU")
    N, R, C = _workers_of(x, (weight, dweight, dbias))
    _like(dy, x, "dy")
    if N == 1 and dy.dim() == 3 and x.shape[0] and not dy.is_contiguous():
        N, R = x.shape[0], x.shape[1]                          # one weight for all: any split of the rows will do
    ptype, pcode = _param_type(weight, dweight, dbias)
    w, dw, db = _param(weight, ptype, device), _param(dweight, ptype, device), _param(dbias, ptype, device)
    lead = x.shape[:-1]
    for s in (mean, rstd):
        if s.dtype != torch.float32 or s.get_device() != device or s.shape != lead or not s.is_contiguous():
            raise TypeError("mean and rstd must be what liec_layer_norm returned")
    if not need_dx:
        dx = None
    elif dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _like(dx, x, "dx")
    ws, need = None, 0
    if dw is not None or db is not None:
        need = lib().liec_layer_norm_workspace(N, R, C)
        if need < 0:
            raise ValueError(f"{N} workers of {R} rows of {C} columns are more than the library takes")
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    _call("liec_layer_norm_backward", device, _rows(dy, N, R, C, "dy"), _rows(x, N, R, C, "x"), mean.data_ptr(), rstd.data_ptr(), w,
          None if dx is None else _rows(dx, N, R, C, "dx"), dw, db, N, R, C, code, pcode, _optional(ws), need)
    return dx
