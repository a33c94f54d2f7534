"""Binding of include/liec_train.h: the operators around the backward pass whose gradients a compressed step takes.

Tensors of N workers carry the workers as their leading dimension.  Every function enqueues its kernels on torch's
current stream of the tensors' device and returns; scratch comes from torch's allocator.  Only arguments are checked and
marshalled here.
"""
from __future__ import annotations

import ctypes
import math
from array import array
from typing import Optional, Sequence, Tuple

import torch

from .binding import _check, lib

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_dtype_code = _DTYPES.get


def _stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _on(device: int):
    """The device of the tensors is the current one while a function launches."""
    return torch.cuda.device(device)


# ---- gradients ------------------------------------------------------------------------------------------------------
def _grad_table(grads: Sequence[torch.Tensor], N: int, whole: bool, device: int) -> array:
    """liec_grad_tensor of each tensor, as the words the struct is made of."""
    words = []
    add = words.extend
    for t in grads:
        code = _dtype_code(t.dtype)
        if code is None or t.get_device() != device:
            raise TypeError("gradients must be float32, bfloat16 or float16 tensors on one GPU")
        count = t.numel()
        if whole:
            if not t.is_contiguous():
                raise ValueError("gradients of one worker must be contiguous")
            add((t.data_ptr(), count, count, code))
            continue
        if t.dim() == 0 or t.shape[0] != N:
            raise ValueError(f"a gradient has shape {tuple(t.shape)}, expected {N} workers as its leading dimension")
        count //= N
        if t.is_contiguous():
            add((t.data_ptr(), count, count, code))
        else:
            if not t[0].is_contiguous():
                raise ValueError("the gradients of a worker must be contiguous within each tensor")
            add((t.data_ptr(), count, t.stride(0), code))
    return array("q", words)


def _grad_args(grads, norms, workers):
    """(tensors' table, its length, N, device, workspace, its bytes)"""
    if not grads and norms is None:
        raise ValueError("no gradients, and no norms to tell the number of workers")
    first = grads[0] if grads else norms
    device = first.get_device()
    if device < 0:
        raise TypeError("gradients must be on the GPU")
    if norms is not None:
        if norms.dtype != torch.float32 or norms.get_device() != device or norms.dim() != 1 or not norms.is_contiguous():
            raise TypeError("norms must be a contiguous float32 vector on the gradients' GPU")
    if workers is not None and workers != 1:
        raise ValueError("workers is 1 for tensors of one worker, or None for tensors with a leading dimension of workers")
    N = 1 if workers == 1 else norms.shape[0] if norms is not None else first.shape[0] if first.dim() else 0
    if norms is not None and norms.shape[0] != N:
        raise ValueError(f"norms has {norms.shape[0]} values, expected {N}")
    table = _grad_table(grads, N, workers == 1, device)
    need = int(lib().liec_grads_workspace(N, len(grads)))
    if need < 0:
        raise ValueError(f"{len(grads)} tensors of {N} workers are more than the library takes")
    return table, len(grads), N, device, torch.empty(need, dtype=torch.uint8, device=first.device), need


def _optional(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def liec_grad_norm(grads: Sequence[torch.Tensor], norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> torch.Tensor:
    """Global l2 norm of each worker's gradients over all tensors, [N] float32, summed in 64 bits.  `workers=1`: the
    tensors, of any shape, belong to one worker; otherwise their leading dimension is the workers'."""
    table, T, N, device, ws, need = _grad_args(grads, norms, workers)
    if norms is None:
        norms = torch.empty(N, dtype=torch.float32, device=grads[0].device)
    with _on(device):
        _check(lib().liec_grad_norm(table.buffer_info()[0], T, N, norms.data_ptr(), ws.data_ptr(), need, _stream(device)), "liec_grad_norm")
    return norms


def liec_clip_grads(grads: Sequence[torch.Tensor], max_norm: float, norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> None:
    """Scales each worker's gradients in place so that their global norm is at most max_norm; `norms`, when given,
    receives the norms before that."""
    table, T, N, device, ws, need = _grad_args(grads, norms, workers)
    with _on(device):
        _check(lib().liec_clip_grads(table.buffer_info()[0], T, N, max_norm, _optional(norms), ws.data_ptr(), need, _stream(device)),
               "liec_clip_grads")


def liec_gather_grads(grads: Sequence[torch.Tensor], rows: torch.Tensor, max_norm: float = math.inf, norms: Optional[torch.Tensor] = None,
                      workers: Optional[int] = None) -> None:
    """Puts each worker's tensors one after the other into its row of `rows` ([N, d] float32, as LiecContext.step reads
    it), scaled so that the row's norm is at most max_norm."""
    table, T, N, device, ws, need = _grad_args(grads, norms, workers)
    total = sum(table[1::4])
    if rows.dtype != torch.float32 or rows.get_device() != device or rows.dim() != 2 or (rows.shape[1] > 1 and rows.stride(1) != 1):
        raise TypeError("rows must be a float32 [N, d] tensor on the gradients' GPU whose rows are contiguous")
    if rows.shape[0] != N or rows.shape[1] != total:
        raise ValueError(f"rows has shape {tuple(rows.shape)}, expected {(N, total)}")
    with _on(device):
        _check(lib().liec_gather_grads(table.buffer_info()[0], T, N, rows.data_ptr(), rows.stride(0), max_norm, _optional(norms), ws.data_ptr(),
                                       need, _stream(device)), "liec_gather_grads")


# ---- layer normalisation --------------------------------------------------------------------------------------------
class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class _Param(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


def _workers_of(x: torch.Tensor, params) -> Tuple[int, int, int]:
    """(N, R, C) of activations x under these weights, biases and their gradients (some of them None)."""
    if x.dim() == 0 or x.shape[-1] < 1:
        raise ValueError(f"activations of shape {tuple(x.shape)} have no columns")
    C = x.shape[-1]
    per_worker = 0
    for p in params:
        if p is None:
            continue
        if p.dim() not in (1, 2) or p.shape[-1] != C or (C > 1 and p.stride(-1) != 1):
            raise ValueError(f"a weight or bias of shape {tuple(p.shape)} does not fit {C} columns, or its columns are not contiguous")
        if p.dim() == 2:
            if x.dim() < 2 or p.shape[0] != x.shape[0] or not p.shape[0]:
                raise ValueError(f"weights of {p.shape[0]} workers do not fit activations of shape {tuple(x.shape)}")
            per_worker = p.shape[0]
    if per_worker:
        return per_worker, x.numel() // (per_worker * C), C
    if x.dim() == 3 and not x.is_contiguous() and x.shape[0]:
        return x.shape[0], x.shape[1], C
    return 1, x.numel() // C, C


def _rows(t: torch.Tensor, N: int, R: int, C: int, like: torch.Tensor, what: str) -> _Rows:
    if t.dtype != like.dtype or t.get_device() != like.get_device():
        raise TypeError(f"{what} must have the activations' type and device")
    if t.shape != like.shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(like.shape)}")
    if t.is_contiguous():
        return _Rows(t.data_ptr(), R * C, C)
    try:
        v = t.view(N, R, C)
    except RuntimeError:
        raise ValueError(f"{what} of strides {t.stride()} is not {N} workers' rows at equal distances") from None
    if C > 1 and v.stride(2) != 1:
        raise ValueError(f"the columns of {what} must be contiguous")
    return _Rows(t.data_ptr(), v.stride(0), v.stride(1))


def _param(p: Optional[torch.Tensor], like: Optional[torch.Tensor], x: torch.Tensor) -> Optional[_Param]:
    if p is None:
        return None
    if p.get_device() != x.get_device() or p.dtype != like.dtype or _dtype_code(p.dtype) is None:
        raise TypeError("weights, biases and their gradients must be float32, bfloat16 or float16, of one type, on the activations' GPU")
    return _Param(p.data_ptr(), p.stride(0) if p.dim() == 2 else 0)


def _ref(s):
    return None if s is None else ctypes.byref(s)


def _activations_type(x: torch.Tensor) -> int:
    code = _dtype_code(x.dtype)
    if code is None or not x.is_cuda:
        raise TypeError("activations must be float32, bfloat16 or float16 on the GPU")
    return code


def liec_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Layer normalisation over the last dimension: (y, mean, rstd), the latter two float32 of x's other dimensions.
    weight and bias: [C], or [N, C] for the N workers of x's leading dimension (columns of a models tensor, say).
    `out` may be x."""
    code = _activations_type(x)
    N, R, C = _workers_of(x, (weight, bias))
    like = weight if weight is not None else bias
    w, b = _param(weight, like, x), _param(bias, like, x)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    xr = _rows(x, N, R, C, x, "x")
    yr = _rows(y, N, R, C, x, "out")
    device = x.get_device()
    with _on(device):
        _check(lib().liec_layer_norm(ctypes.byref(xr), _ref(w), _ref(b), ctypes.byref(yr), mean.data_ptr(), rstd.data_ptr(), N, R, C, eps, code,
                                     0 if like is None else _DTYPES[like.dtype], _stream(device)), "liec_layer_norm")
    return y, mean, rstd


def liec_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                             dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             need_dx: bool = True) -> Optional[torch.Tensor]:
    """Gradients of liec_layer_norm: returns dx (a new tensor unless one is given, which may be dy or x; None with
    need_dx=False) and writes the gradients of weight and bias into dweight and dbias where they are given: [N, C] takes
    each worker's own sum (columns of the gradient rows of a step, say), [C] the sum over everything."""
    code = _activations_type(x)
    N, R, C = _workers_of(x, (weight, dweight, dbias))
    like = weight if weight is not None else dweight if dweight is not None else dbias
    if N == 1 and not dy.is_contiguous() and dy.dim() == 3 and dy.shape == x.shape and x.shape[0]:
        N, R = x.shape[0], x.shape[1]                          # one weight for all: any split of the rows will do
    w, dw, db = _param(weight, like, x), _param(dweight, like, x), _param(dbias, like, x)
    for s in (mean, rstd):
        if s.dtype != torch.float32 or s.get_device() != x.get_device() or s.shape != x.shape[:-1] or not s.is_contiguous():
            raise TypeError("mean and rstd must be what liec_layer_norm returned")
    if not need_dx:
        dx = None
    elif dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    gr, xr = _rows(dy, N, R, C, x, "dy"), _rows(x, N, R, C, x, "x")
    dr = None if dx is None else _rows(dx, N, R, C, x, "dx")
    device = x.get_device()
    ws, need = None, 0
    if dw is not None or db is not None:
        need = int(lib().liec_layer_norm_workspace(N, R, C))
        if need < 0:
            raise ValueError(f"{N} workers of {R} rows of {C} columns are more than the library takes")
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    with _on(device):
        _check(lib().liec_layer_norm_backward(ctypes.byref(gr), ctypes.byref(xr), mean.data_ptr(), rstd.data_ptr(), _ref(w), _ref(dr), _ref(dw),
                                              _ref(db), N, R, C, code, 0 if like is None else _DTYPES[like.dtype], _optional(ws), need,
                                              _stream(device)), "liec_layer_norm_backward")
    return dx
