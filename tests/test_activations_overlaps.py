"""Operands of the operators on activations that lie between one another, for any number of workers: checks that need no GPU."""
import itertools
import os
import random
import sys
import time

import pytest

sys.path.insert(0, os.path.dirname(__file__))
from test_activations_abi import EINVAL, Call, Images, Saved, calls, fakes  # noqa: E402,F401
from test_train_abi import Param, lib  # noqa: E402,F401


def far_apart(calls, N):  # noqa: F811
    """A valid call whose operands have room for any number of workers."""
    c = Call(calls, N=N)
    at = iter(range(1 << 44, 1 << 45, 1 << 34))
    image = (c.B * c.S * c.C, c.S * c.C, c.C)
    c.x, c.y, c.dy, c.dx = (Images(next(at), *image) for _ in range(4))
    c.w, c.b, c.dw, c.db = (Param(next(at), c.C) for _ in range(4))
    c.mean, c.rstd, c.ws = (next(at) for _ in range(3))
    c.saved = Saved(next(at), next(at))
    assert c.forward() != EINVAL and c.backward() != EINVAL
    return c


@fakes
@pytest.mark.parametrize("N", [3, 2048, 2049, 5000, 65_535])
def test_images_cut_out_of_wider_ones(calls, N):  # noqa: F811
    """Images [N, 2, 5, 24] whose workers, images and positions all lie apart: no two distances describe them."""
    c = far_apart(calls, N)
    far = (1000, 200, 30)
    base = 1 << 40
    x = Images(base, *far)
    began = time.perf_counter()
    # behind one another, between one another, at other distances between one another, and the same backwards
    assert c.forward(x=x, y=Images(base + 4000 * N, *far)) != EINVAL
    assert c.forward(x=x, y=Images(base + 1600, *far)) != EINVAL
    assert c.forward(x=x, y=Images(base + 1600, 1000, 180, 36)) != EINVAL
    assert c.forward(x=x, y=Images(base + 1600 + 4000 * (N - 1), -1000, 200, 30)) != EINVAL
    assert c.backward(dy=x, dx=Images(base + 1600, *far)) != EINVAL
    assert c.backward(dy=Images(base, 1000, 200, 31), dx=Images(base + 1600, *far)) != EINVAL
    # the last worker's last position, and one value before it
    assert c.forward(x=x, y=Images(base + 4 * (1000 * (N - 1) + 200 + 4 * 30 + 23), *far)) == EINVAL
    assert c.forward(x=x, y=Images(base + 4 * (1000 * (N - 1) + 200 + 4 * 30 + 24), *far)) != EINVAL
    assert c.forward(x=x, y=Images(base + 800, *far)) == EINVAL
    assert c.forward(x=x, y=Images(base + 1600 + 4 * 1000 * (N - 1), -1000, 200, 6)) == EINVAL
    assert c.backward(dy=x, dx=Images(base + 800, *far)) == EINVAL
    # the workers' parameters and statistics between the images
    assert c.forward(x=Images(1 << 42, *far), y=Images((1 << 42) + 1600, *far), mean=(1 << 42) + 4 * 224) == EINVAL
    assert time.perf_counter() - began < 2.0


@fakes
def test_one_workers_images_for_all(calls):  # noqa: F811
    c = far_apart(calls, 5000)
    x = Images(1 << 40, 0, 200, 30)                          # seen 5000 times
    assert c.forward(x=x, y=Images((1 << 40) + 4 * 400, 1000, 200, 30)) != EINVAL
    assert c.forward(x=x, y=Images((1 << 40) + 4 * 300, 1000, 200, 30)) == EINVAL
    assert c.forward(x=x, y=Images((1 << 40) - 4 * 1000 * 4999, 1000, 200, 30)) == EINVAL


@fakes
@pytest.mark.parametrize("N", [3, 5000])
def test_images_of_any_order_in_memory(calls, N):  # noqa: F811
    """Workers, images and positions in any order, with room between all of them and other images in their rows."""
    c = far_apart(calls, N)
    sizes = {"worker": N, "image": c.B, "row": c.S}
    base = 1 << 40
    began = time.perf_counter()
    for gap in (0, 1):
        for order in itertools.permutations(sizes):          # the innermost first
            strides, room = {}, 70
            for name in order:
                strides[name] = room
                room = room * sizes[name] + 100 * gap
            at = lambda to, sign=1: Images(base + 4 * to + (0 if sign > 0 else 4 * (N - 1) * strides["worker"]), sign * strides["worker"], strides["image"], strides["row"])  # noqa: E731
            last = sum(strides[name] * (sizes[name] - 1) for name in sizes)
            x = at(0)
            for sign in (1, -1):
                assert c.forward(x=x, y=at(24, sign)) != EINVAL and c.forward(x=x, y=at(46, sign)) != EINVAL and c.forward(x=x, y=at(room, sign)) != EINVAL
                assert c.forward(x=x, y=at(23, sign)) == EINVAL and c.forward(x=x, y=at(47, sign)) == EINVAL
                assert c.backward(dy=x, dx=at(40, sign)) != EINVAL and c.backward(dy=x, dx=at(10, sign)) == EINVAL
            assert c.forward(x=x, y=Images(base + 4 * (last + 24), 240, 120, 24)) != EINVAL
            assert c.forward(x=x, y=Images(base + 4 * (last + 23), 240, 120, 24)) == EINVAL
            assert c.forward(x=x, mean=base + 4 * (last + 23)) == EINVAL and c.forward(x=x, w=None, b=None, rstd=base + 4 * (last + 24)) != EINVAL
    assert time.perf_counter() - began < 10.0


@fakes
def test_against_every_byte(calls):  # noqa: F811
    """Small images at random distances, overlapping and not: as the sets of their bytes say."""
    rng = random.Random(5)
    N, B, S, C = 3, 2, 4, 3
    met = apart = 0
    c = Call(calls, N=N, B=B, S=S, C=C, G=1)
    base = 1 << 40

    def values(m):
        return {(m.data - base) // 4 + i * m.worker_stride + j * m.image_stride + k * m.row_stride + ch for i in range(N) for j in range(B) for k in range(S) for ch in range(C)}

    for _ in range(4000):
        strides = [rng.choice((1, -1)) * rng.randrange(0, 60) for _ in range(3)]
        x = Images(base, *strides)
        out = [3, 13, 27]
        rng.shuffle(out)
        y = Images(base + 4 * rng.randrange(-150, 150), *(rng.choice((1, -1)) * s for s in out))
        if len(values(y)) != N * B * S * C:
            continue
        share = bool(values(x) & values(y))
        same = (x.data, x.worker_stride, x.image_stride, x.row_stride) == (y.data, y.worker_stride, y.image_stride, y.row_stride)
        assert (c.forward(x=x, y=y) == EINVAL) == (share and not same), (strides, out)
        met, apart = met + share, apart + (not share)
    assert met > 100 and apart > 100
