"""Clipping tensors that lie between one another in memory without sharing any of it."""
import ctypes
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import U32, assert_within, generator  # noqa: E402
from test_train_abi import Tensor  # noqa: E402

pytestmark = GPU_MARKS


def _clip(buffer, spans, N, share=0.5):
    """Clips spans (start, count, stride of the workers, in values) of an fp32 buffer, and checks norms, what was scaled and that
    nothing else was touched."""
    import paper_2402_11857_amd as pkg

    lib = pkg.lib()
    at = [[torch.arange(s + i * stride, s + i * stride + n, device=DEV) for s, n, stride in spans] for i in range(N)]
    index = [torch.cat(a) for a in at]
    assert torch.cat(index).unique().numel() == sum(a.numel() for a in index)          # none shared
    before = buffer.clone()
    want = torch.stack([before[a].double().norm() for a in index])
    bound = float(want.min()) * share
    arr = (Tensor * len(spans))(*[Tensor(buffer.data_ptr() + 4 * s, n, stride, 0, 0) for s, n, stride in spans])
    need = lib.liec_grads_workspace(N, len(spans))
    ws, norms = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty(N, device=DEV)
    status = lib.liec_clip_grads(ctypes.byref(arr), len(spans), N, bound, norms.data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    assert_within(norms, want, want * (U32 + 1e-12), "norms")
    expect = before.double()
    for i, a in enumerate(index):
        expect[a] *= bound / want[i]
    assert_within(buffer, expect, expect.abs() * 3 * U32 + 2.0 ** -149, "values")
    rest = torch.ones_like(buffer, dtype=torch.bool)
    for a in index:
        rest[a] = False
    assert torch.equal(buffer[rest], before[rest])


def _matrix(N, D, seed):
    return torch.randn(N * D, generator=generator(seed), device=DEV)


def test_columns_with_workers_in_reverse():
    say("case clip, columns of a matrix, workers in reverse")
    N, D = 3, 40
    _clip(_matrix(N, D, 301), [((N - 1) * D, 10, -D), ((N - 1) * D + 10, 10, -D), ((N - 1) * D + 30, 7, -D)], N)
    _clip(_matrix(N, D, 302), [((N - 1) * D, 10, -D), (10, 10, D)], N)                 # one of them in order


def test_columns_that_wrap_around_their_rows():
    say("case clip, columns that begin in one row and end in the next")
    _clip(_matrix(4, 100, 303), [(90, 20, 100), (10, 30, 100), (45, 45, 100)], 3)


def test_distances_that_differ():
    import paper_2402_11857_amd as pkg

    say("case clip, tensors at distances that differ")
    _clip(_matrix(4, 64, 306), [(0, 64, 64), (192, 20, 20)], 3)                        # a tensor behind the matrix's last row
    _clip(_matrix(4, 64, 307), [(0, 50, 64), (50, 4, 4)], 3)                           # and one in a gap of its columns
    rows = torch.ones(8, 64, device=DEV)
    with pytest.raises(pkg.LiecError):                       # between one another: counts as sharing
        pkg.liec_clip_grads([rows[:4, :16], rows[::2, 16:32]], 1.0)
    assert bool((rows == 1).all())


def test_a_matrix_and_a_tensor_of_its_own():
    say("case clip, 4000 columns of a matrix and another tensor, 8 workers")
    import time

    import paper_2402_11857_amd as pkg

    N, T = 8, 4000
    rows = torch.randn(N, 2 * T, generator=generator(307), device=DEV)
    views = [rows[:, 2 * i:2 * i + 1] for i in range(T)]
    other = torch.randn(N, 33, generator=generator(308), device=DEV)
    pkg.liec_clip_grads(views, 1e9)
    torch.cuda.synchronize()

    def host(tensors):
        best = 1e9
        for _ in range(5):
            t = time.perf_counter()
            pkg.liec_clip_grads(tensors, 1e9)
            best = min(best, time.perf_counter() - t)
            torch.cuda.synchronize()
        return best

    alone, both = host(views), host(views + [other])
    assert both < 4 * alone, (alone, both)                   # comparing every pair took 41 ms, 20 times as long


def test_tensors_that_do_share_memory_are_refused():
    import paper_2402_11857_amd as pkg

    say("case clip, tensors that share memory")
    rows = torch.ones(4, 64, device=DEV)
    flat = rows.view(-1)
    for bad in ([rows[:, :10], rows[:, 9:20]],
                [flat[:192].view(3, 64)[:, 50:], flat[64:].view(3, 64)[:, :1], flat[32:224].view(3, 64)[:, 20:40]],
                [flat[:128].view(2, 64)[:, :16], flat[64:96].view(2, 16)]):
        with pytest.raises(pkg.LiecError):
            pkg.liec_clip_grads(bad, 1.0)
    assert bool((rows == 1).all())
