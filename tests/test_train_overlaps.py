"""include/liec_train.h: what one kernel writes while others read or write it must be memory of its own.  The checks look at
addresses only; a call that they let through fails here for want of a GPU with another status than LIEC_EINVAL."""
import ctypes
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
from test_train_abi import Tensor, lib  # noqa: E402,F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="passes addresses that no memory stands behind")
MB = 1 << 20
EINVAL = 1


def _grads(lib, name, tensors, N, norms, ws, rows=None, stride=0, bound=1.0):
    arr = (Tensor * len(tensors))(*[Tensor(*t, 0) for t in tensors])
    need = lib.liec_grads_workspace(N, len(tensors))
    if name == "norm":
        return lib.liec_grad_norm(arr, len(tensors), N, norms, ws, need, None)
    if name == "clip":
        return lib.liec_clip_grads(arr, len(tensors), N, bound, norms, ws, need, None)
    return lib.liec_gather_grads(arr, len(tensors), N, rows, stride, bound, norms, ws, need, None)


def test_norms_and_scratch_of_the_gradient_operators(lib):  # noqa: F811
    N = 3
    a, b, rows, norms, ws = (MB * k for k in (1, 2, 3, 4, 5))
    tensors = [(a, 1000, 1000, 0), (b, 77, 100, 1)]          # the second has gaps of 46 bytes
    need = lib.liec_grads_workspace(N, 2)

    def refused(name, norms, ws, **kw):
        return _grads(lib, name, tensors, N, norms, ws, rows=rows, stride=1080, **kw) == EINVAL

    for name in ("norm", "clip", "gather"):
        assert not refused(name, norms, ws)
        assert refused(name, ws + 16, ws)                    # norms in the scratch
        assert refused(name, ws + need - 4, ws) and not refused(name, ws + need, ws)
        assert refused(name, norms, a + 11_984)              # scratch in a tensor
        assert refused(name, norms, a - need + 16) and not refused(name, norms, a - need)
    for name in ("clip", "gather"):
        assert refused(name, a + 11_996, ws) and not refused(name, a + 12_000, ws)
        assert refused(name, b + 152, ws) and refused(name, b + 192, ws)
        assert not refused(name, b + 156, ws)                # 12 bytes in the gap
        assert refused(name, a, ws, bound=float("inf"))
    assert not refused("norm", a, ws)                        # written after everything has been read
    assert refused("gather", rows + 4 * 1076, ws)            # in worker 0's row
    assert not refused("gather", rows + 4 * 1077, ws)        # between the first two
    assert refused("gather", norms, rows + 16)               # scratch in the rows
    assert not refused("gather", None, rows + 16, bound=float("inf"))     # scratch that is not used
