"""Workers whose gradients exceed 256 MB each, which are squared and scaled one after the other."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, TINY, U, U32, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS
MB256 = 256 << 20


def _case(N, dtype, strided, many):
    """Tensors of N workers, more than 256 MB a worker; the workers' values differ in size."""
    size = torch.empty(0, dtype=DTYPES[dtype]).element_size()
    small = [1 + 131 * i for i in range(300)] if many else [77]
    counts = small[:150] + [MB256 // size + 4099] + small[150:]
    gen = generator(401)
    worker = torch.tensor([1.0, 3.0, 0.25], device=DEV)[:N, None]
    if strided:                                              # columns of a matrix with a gap after each
        rows = torch.empty(N, sum(counts) + len(counts), dtype=DTYPES[dtype], device=DEV)
        at, tensors = 0, []
        for n in counts:
            tensors.append(rows[:, at:at + n])
            at += n + 1
    else:
        tensors = [torch.empty(N, n, dtype=DTYPES[dtype], device=DEV) for n in counts]
    for i, t in enumerate(tensors):
        t.normal_(generator=gen).mul_(worker * (0.01 if t.shape[1] > 1_000_000 else 10.0))
        t[:, 0] = 0.5 + i % 7                                # both ends are there to be seen
        t[:, -1] = -0.25 - i % 5
    return tensors


def _norms(tensors, N):
    total = torch.zeros(N, dtype=torch.float64, device=DEV)
    for t in tensors:
        for i in range(N):
            total[i] += torch.linalg.vector_norm(t[i].double()) ** 2
    return total.sqrt()


@pytest.mark.parametrize("N,dtype,strided,many", [(2, "fp32", False, False), (3, "bf16", False, True), (3, "bf16", True, True), (2, "fp16", True, False)])
def test_workers_one_after_the_other(N, dtype, strided, many):
    import paper_2402_11857_amd as pkg

    say(f"case gradients of more than 256 MB, {N} workers, {dtype}{', strided' if strided else ''}{', 301 tensors' if many else ''}")
    tensors = _case(N, dtype, strided, many)
    want = _norms(tensors, N)
    bound = float(want.sort().values[:2].mean())             # between the two smallest: one worker stays as it is
    factor = torch.where(want <= bound, torch.ones_like(want), bound / want)
    assert int((factor == 1).sum()) == 1
    d = sum(t.shape[1] for t in tensors)
    rows, norms = torch.empty(N, d + 3, device=DEV), torch.full((N,), -1.0, device=DEV)
    rows[:, d:] = 7.0
    pkg.liec_gather_grads(tensors, rows[:, :d], bound, norms)
    assert_within(norms, want, want * (U32 + 1e-12), "norms of the gather")
    before = [t.clone() for t in tensors]
    norms.fill_(-1.0)
    pkg.liec_clip_grads(tensors, bound, norms)
    assert_within(norms, want, want * (U32 + 1e-12), "norms of the clip")
    assert bool((rows[:, d:] == 7.0).all())
    u, at = U[dtype], 0
    for k, (t, b) in enumerate(zip(tensors, before)):
        for i in range(N):
            value = b[i].double() * factor[i]
            assert_within(rows[i, at:at + t.shape[1]], value, value.abs() * 3 * U32 + 2.0 ** -149, f"row {i}, tensor {k}")
            assert_within(t[i], value, value.abs() * (3 * U32 + (1.01 * u if u > U32 else 0.0)) + TINY[dtype], f"worker {i}, tensor {k}")
            if factor[i] == 1.0:
                assert torch.equal(t[i], b[i])
        at += t.shape[1]
