"""The operators around the backward pass whose gradients a compressed step takes (include/liec_train.h).

Tensors of N workers carry the workers as their leading dimension.  Every function enqueues its kernels on torch's current
stream of the tensors' device and returns; scratch comes from torch's allocator.  Arguments are checked and marshalled by
the compiled module ``_train.so``: TypeError for types and devices, ValueError for shapes and strides, LiecError for what
the library refuses.  There is no CPU fallback.

The functions are not differentiable: results carry no history, whether or not the operands require a gradient, so call
liec_layer_norm_backward for one.  Tensors that a function writes to count as changed in place, so automatic
differentiation notices where it had saved their values.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence, Tuple

import torch

from . import binding

_ENTRY_POINTS = ("liec_grads_workspace", "liec_grad_norm", "liec_clip_grads", "liec_gather_grads", "liec_layer_norm",
                 "liec_layer_norm_workspace", "liec_layer_norm_backward")
_native = _bound_to = None


def _stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def native():
    """The compiled module, given the entry points of the loaded library; raises if either is absent."""
    global _native, _bound_to
    library = binding.lib()
    if _bound_to is not library:
        try:
            from . import _train
        except ImportError as e:
            raise RuntimeError(f"{os.path.join(os.path.dirname(__file__), '_train.so')} cannot be loaded ({e}): build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`. There is no fallback path.") from None
        addresses = [ctypes.cast(getattr(library, name), ctypes.c_void_p).value for name in _ENTRY_POINTS]
        # the current stream's handle without an object for the stream (1 us of a call), where torch has it
        _train.bind(binding.LiecError, getattr(torch._C, "_cuda_getCurrentRawStream", _stream), *addresses)
        _native, _bound_to = _train, library
    return _native


def _whole(workers: Optional[int]) -> bool:
    if workers is not None and workers != 1:
        raise ValueError("workers is 1 for tensors of one worker, or None for tensors with a leading dimension of workers")
    return workers == 1


def liec_grad_norm(grads: Sequence[torch.Tensor], norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> torch.Tensor:
    """Global l2 norm of each worker's gradients over all tensors, [N] float32, summed in 64 bits.  `workers=1`: the
    tensors, of any shape, belong to one worker; otherwise their leading dimension is the workers'."""
    return native().grad_norm(grads, norms, _whole(workers))


def liec_clip_grads(grads: Sequence[torch.Tensor], max_norm: float, norms: Optional[torch.Tensor] = None, workers: Optional[int] = None) -> None:
    """Scales each worker's gradients in place so that their global norm is at most max_norm; `norms`, when given,
    receives the norms before that."""
    native().clip_grads(grads, max_norm, norms, _whole(workers))


def liec_gather_grads(grads: Sequence[torch.Tensor], rows: torch.Tensor, max_norm: float = math.inf, norms: Optional[torch.Tensor] = None,
                      workers: Optional[int] = None) -> None:
    """Puts each worker's tensors one after the other into its row of `rows` ([N, d] float32, as LiecContext.step reads
    it), scaled so that the row's norm is at most max_norm."""
    native().gather_grads(grads, rows, max_norm, norms, _whole(workers))


def liec_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Layer normalisation over the last dimension: (y, mean, rstd), the latter two float32 of x's other dimensions.
    weight and bias: [C], or [N, C] for the N workers of x's leading dimension (columns of a models tensor, say).
    `out` may be x."""
    return native().layer_norm(x, weight, bias, eps, out)


def liec_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                             dx: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                             need_dx: bool = True) -> Optional[torch.Tensor]:
    """Gradients of liec_layer_norm: returns dx (a new tensor unless one is given, which may be dy or x; None with
    need_dx=False) and writes the gradients of weight and bias into dweight and dbias where they are given: [N, C] takes
    each worker's own sum (columns of the gradient rows of a step, say), [C] the sum over everything."""
    return native().layer_norm_backward(dy, x, mean, rstd, weight, dx, dweight, dbias, bool(need_dx))
