"""include/liec_train.h: what one kernel writes while others read or write it must be memory of its own.  The checks look at
addresses only; a call that they let through fails here for want of a GPU with another status than LIEC_EINVAL."""
import ctypes
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
from test_train_abi import Param, Rows, Tensor, lib  # noqa: E402,F401

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


class _LayerNorm:
    """Calls on fp32 operands of N x R rows of C columns, each at an address of its own unless one is given."""

    def __init__(self, lib, N, R, C):  # noqa: F811
        self.lib, self.N, self.R, self.C = lib, N, R, C
        self.need = lib.liec_layer_norm_workspace(N, R, C)

    def rows(self, k):
        return Rows(k * MB, self.R * self.C, self.C)

    def forward(self, x=None, y=None, w=None, b=None, mean=7 * MB, rstd=8 * MB):
        ref, x, y = ctypes.byref, x or self.rows(1), y or self.rows(2)
        w, b = w or Param(5 * MB, self.C), b or Param(6 * MB, self.C)
        return self.lib.liec_layer_norm(ref(x), ref(w), ref(b), ref(y), mean, rstd, self.N, self.R, self.C, 1e-5, 0, 0, None)

    def backward(self, dy=None, x=None, dx=None, w=None, dw=None, db=None, mean=7 * MB, rstd=8 * MB, ws=11 * MB, ptype=0):
        ref, dy, x, dx = ctypes.byref, dy or self.rows(1), x or self.rows(2), dx or self.rows(3)
        w, dw, db = w or Param(5 * MB, self.C), dw or Param(9 * MB, self.C), db or Param(10 * MB, self.C)
        return self.lib.liec_layer_norm_backward(ref(dy), ref(x), mean, rstd, ref(w), ref(dx), ref(dw), ref(db), self.N, self.R, self.C, 0, ptype, ws,
                                                 self.need, None)


def test_rows_that_are_written_and_rows_that_are_read(lib):  # noqa: F811
    N, R, C, S = 3, 10, 64, 200
    f = _LayerNorm(lib, N, R, C)
    assert f.forward() != EINVAL and f.backward() != EINVAL

    def wide(column, row=0, s=S):                            # columns of a matrix of s values a row
        return Rows(12 * MB + 4 * (row * s + column), R * s, s)

    for a, b, meet in ((wide(0), wide(64), False), (wide(0), wide(63), True), (wide(64), wide(0), False), (wide(3), wide(0), True),
                       (wide(0, 1), wide(0), True), (wide(0, 1), wide(64), False), (wide(0, 1), wide(137), True), (wide(0, 1), wide(136), False),
                       (wide(0, N * R), wide(0), False), (wide(0, N * R - 1), wide(0), True),
                       (wide(0), Rows(12 * MB + 4 * 64, R * S + S, S), False),               # one distance differs
                       (wide(0), Rows(12 * MB + 4 * 64, R * S + S - 1, S), True),
                       (wide(0), Rows(12 * MB + 4 * 64, R * S, 2 * S), False),               # rows of a worker reach the next one's
                       (wide(0), Rows(12 * MB + 4 * 64, 2 * R * S, 2 * S), False),
                       (wide(0), Rows(12 * MB + 4 * 64, 2 * R * S, 2 * S + 30), True),
                       (wide(0), Rows(12 * MB + 4 * ((N * R - 1) * S), -R * S, -S), True),   # the same rows in reverse
                       (wide(0), Rows(12 * MB + 4 * ((N * R - 1) * S + 64), -R * S, -S), False)):
        assert (f.forward(x=b, y=a) == EINVAL) == meet
        assert (f.backward(dy=b, dx=a) == EINVAL) == meet
        assert (f.backward(x=b, dx=a) == EINVAL) == meet
    # in place, with distances that nothing is counted with
    one = _LayerNorm(lib, 1, R, C)
    assert one.forward(x=Rows(MB, 0, S), y=Rows(MB, 77, S)) != EINVAL
    assert one.forward(x=Rows(MB, 0, S), y=Rows(MB, 0, S + 1)) == EINVAL
    row = _LayerNorm(lib, N, 1, C)
    assert row.backward(dy=Rows(MB, S, 0), dx=Rows(MB, S, 5)) != EINVAL


def test_weight_gradients(lib):  # noqa: F811
    N, R, C, S = 3, 10, 64, 200
    f = _LayerNorm(lib, N, R, C)
    at = Param(13 * MB, S)
    for column, meet in ((0, True), (63, True), (64, False), (136, False), (137, True), (199, True), (200, True), (N * S, False), (-64, False), (-63, True)):
        assert (f.backward(dw=at, db=Param(13 * MB + 4 * column, S)) == EINVAL) == meet, column
        assert (f.backward(dw=Param(13 * MB + 4 * column, S), db=at) == EINVAL) == meet, column
        assert (f.backward(dw=Param(13 * MB + 4 * column, S), w=at) == EINVAL) == (meet and column != 0), column     # w itself may be replaced
        assert (f.backward(db=Param(13 * MB + 4 * column, S), w=at) == EINVAL) == (meet and column != 0), column
    assert f.backward(dw=Param(9 * MB + 4 * 64, -S), db=Param(9 * MB, S)) != EINVAL
    assert f.backward(dw=Param(9 * MB, C), w=Param(9 * MB, 0)) == EINVAL                     # a shared weight in one worker's gradient
    assert f.backward(dw=Param(9 * MB, 0), db=Param(9 * MB + 4 * 63, 0)) == EINVAL
    assert f.backward(dw=Param(9 * MB, 0), db=Param(9 * MB + 4 * 64, 0)) != EINVAL
    for place in ("dy", "x", "dx", "mean", "rstd"):
        k = {"dy": 1, "x": 2, "dx": 3, "mean": 7, "rstd": 8}[place]
        size = 4 * N * R * (C if k < 4 else 1)
        for start, meet in ((k * MB, True), (k * MB + size - 4, True), (k * MB + size, False), (k * MB - 4 * C, False), (k * MB - 4 * C + 4, True)):
            assert (f.backward(dw=Param(start, 0), db=Param(10 * MB, 0)) == EINVAL) == meet, (place, start)
            assert (f.backward(db=Param(start, 0), dw=Param(10 * MB, 0)) == EINVAL) == meet, (place, start)
    empty = _LayerNorm(lib, N, 0, C)
    assert empty.backward(dw=at, db=Param(13 * MB + 4 * 63, S)) == EINVAL


def test_statistics_weights_and_scratch(lib):  # noqa: F811
    N, R, C = 3, 10, 64
    f = _LayerNorm(lib, N, R, C)
    stat, act, par = 4 * N * R, 4 * N * R * C, 4 * N * C

    def places(start, size, own):
        """Starts of an operand of `own` bytes around one of `size` bytes, and whether they meet."""
        return ((start, True), (start + size - 4, True), (start + size, False), (start - own + 4, True), (start - own, False))

    for k, size in ((1, act), (2, act), (5, par), (6, par)):                                 # x, y, weight, bias
        for start, meet in places(k * MB, size, stat):
            assert (f.forward(mean=start) == EINVAL) == meet
            assert (f.forward(rstd=start) == EINVAL) == meet
    for start, meet in places(7 * MB, stat, stat):
        assert (f.forward(rstd=start) == EINVAL) == meet
    assert f.forward(mean=None, rstd=None) != EINVAL
    for start, meet in places(2 * MB, act, par):
        assert (f.forward(w=Param(start, C)) == EINVAL) == meet
        assert (f.forward(b=Param(start, C)) == EINVAL) == meet
    for start, meet in places(3 * MB, act, stat):
        assert (f.backward(mean=start) == EINVAL) == meet
        assert (f.backward(rstd=start) == EINVAL) == meet
    for start, meet in places(3 * MB, act, par):
        assert (f.backward(w=Param(start, C)) == EINVAL) == meet
    assert f.backward(mean=7 * MB, rstd=7 * MB) != EINVAL                                    # only read
    for k, size in ((1, act), (2, act), (3, act), (5, par), (7, stat), (8, stat), (9, par), (10, par)):
        start = k * MB + size & -16                          # scratch begins at multiples of 16
        for ws, meet in ((k * MB, True), (start - 16, True), (start + 16, False), (k * MB - f.need + 16, True), (k * MB - (f.need + 15 & -16), False)):
            assert (f.backward(ws=ws) == EINVAL) == meet, (k, ws - k * MB)
