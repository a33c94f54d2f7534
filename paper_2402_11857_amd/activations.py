"""The operators on activations of N workers (include/liec_activations.h): checkpoints in 8 bits, group normalisation with an
activation function, channels last, and its gradients, and the gradient of a linear layer's weight from a checkpoint.

As in ``train``: tensors of N workers carry the workers as their leading dimension, kernels go to torch's current stream of the
tensors' device, scratch comes from torch's allocator, results carry no history, and tensors that a function writes to count as
changed in place.  TypeError for types and devices, ValueError for shapes and strides, LiecError for what the library refuses.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple, Union

import torch

from . import binding, train

_ENTRY_POINTS = ("liec_checkpoint_save", "liec_checkpoint_load", "liec_group_norm_workspace", "liec_group_norm", "liec_group_norm_backward",
                 "liec_weight_grad_workspace", "liec_weight_grad")
_ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}
_native = _bound_to = None


class Checkpoint(NamedTuple):
    """Activations in 8 bits: every 32 consecutive columns of a row share one of the exponents s, and a value q stands for
    q * 2^(s - 127); s = 255: NaN throughout (columns that held an infinity or a NaN)."""
    values: torch.Tensor          # int8, the activations' shape, contiguous
    exponents: torch.Tensor       # uint8, the same with ceil(columns / 32) columns, contiguous


def native():
    """The compiled module, given the entry points of the loaded library; raises if either is absent."""
    global _native, _bound_to
    library = binding.lib()
    if _bound_to is not library:
        module = train.native()
        module.bind_activations(*(ctypes.cast(getattr(library, name), ctypes.c_void_p).value for name in _ENTRY_POINTS))
        _native, _bound_to = module, library
    return _native


def _activation(name: str) -> int:
    try:
        return _ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation is one of {', '.join(map(repr, _ACTIVATIONS))}, got {name!r}") from None


def liec_checkpoint_save(x: torch.Tensor, out: Optional[Checkpoint] = None) -> Checkpoint:
    """A checkpoint of activations [..., C] (float32, bfloat16, float16): each value rounded to nearest, off by at most 1/127 of the
    largest of its 32 columns.  `out`: an earlier checkpoint of this shape, which is overwritten."""
    return Checkpoint(*native().checkpoint_save(x, out))


def liec_checkpoint_load(saved: Checkpoint, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """What a checkpoint stands for: exact in float32 and bfloat16.  With `out`, in its type."""
    return native().checkpoint_load(saved, dtype, out)


def liec_group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    activation: str = "none", out: Optional[torch.Tensor] = None, save: bool = False) -> Tuple:
    """Group normalisation of images [N, B, ..., C], channels last, over an image's positions and the C / groups neighbouring
    channels of a group, scaled by weight, shifted by bias and passed through an activation function ("none", "relu", "silu"):
    (y, mean, rstd), the latter two float32 [N, B, groups] (NaN for images without positions).  weight and bias: [C], or [N, C] for
    the N workers (columns of a models tensor, say).  `out` may be x.  With save=True a checkpoint of x, written in the same
    pass, comes as the fourth."""
    r = native().group_norm(x, groups, weight, bias, eps, _activation(activation), out, bool(save))
    first = out if out is not None else r[0]
    return (first, r[1], r[2], Checkpoint(r[3], r[4])) if save else (first, r[1], r[2])


def liec_group_norm_backward(dy: torch.Tensor, x: Union[torch.Tensor, Checkpoint], mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                             bias: Optional[torch.Tensor] = None, activation: str = "none", dx: Optional[torch.Tensor] = None,
                             dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, need_dx: bool = True) -> Optional[torch.Tensor]:
    """Gradients of liec_group_norm from its input or a checkpoint of it: returns dx (a new tensor unless one is given, which may be dy
    or x; None with need_dx=False) and writes the gradients of weight and bias into dweight and dbias where they are
    given: [N, C] takes each worker's own sum (columns of the gradient rows of a step, say), [C] the sum over everything."""
    return native().group_norm_backward(dy, x, mean, rstd, weight, bias, _activation(activation), dx, dweight, dbias, bool(need_dx))


def liec_weight_grad(dy: torch.Tensor, saved: Checkpoint, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradients of the weight [O, C] and the bias [O] of a linear layer (a convolution with kernels of 1 x 1, channels last) from dy
    [N, ..., O] and a checkpoint [N, ..., C] of its input: dweight [N, O, C] (a new float32 tensor unless one is given, such
    as columns of the gradient rows of a step) takes each worker's own sum, [O, C] the sum over everything; so does dbias, [N, O]
    or [O], where it is given."""
    return native().weight_grad(dy, saved, dweight, dbias)
