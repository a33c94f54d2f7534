"""Activations that are views: slices of wider rows, rows of another order, under weights that all rows share."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from test_gpu_layer_norm import EPS, _check_backward, _check_forward, _inputs  # noqa: E402

pytestmark = GPU_MARKS


def _shared(shape, seed):
    x, dy, w, b = _inputs(shape, "bf16", seed=seed)
    return x, dy, w[0].clone(), b[0].clone()


def _forward_and_backward(x, dy, w, b, out=None, dx=None):
    import paper_2402_11857_amd as pkg

    y, mean, rstd = pkg.liec_layer_norm(x, w, b, EPS, out=out)
    _check_forward(x, w, b, EPS, y, mean, rstd)
    dw, db = torch.full_like(w, 9.0), torch.full_like(b, 9.0)
    got = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dx=dx, dweight=dw, dbias=db)
    _check_backward(dy, x, mean, rstd, w, got, dw, db)
    assert out is None or y is out
    assert dx is None or got is dx


def test_more_sequences_than_workers():
    say("case layer norm, a slice of 70000 sequences")
    for C in (5, 40):
        x, dy, w, b = _shared((70_000, 2, C + 3), seed=201)
        _forward_and_backward(x[..., :C], dy[..., 1:1 + C], w[:C], b[:C])
        _forward_and_backward(x[..., :C].contiguous(), dy[..., 1:1 + C], w[:C], b[:C])


def test_scratch_of_a_slice_is_that_of_its_rows():
    """The sums of a slice of evenly spaced rows take as much scratch as those of a contiguous tensor."""
    import paper_2402_11857_amd as pkg

    say("case layer norm, scratch of a slice")
    N, R, C = 8192, 8, 256
    x, dy = (torch.ones(N, R, C + 8, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    mean, rstd, dw = torch.zeros(N, R, device=DEV), torch.ones(N, R, device=DEV), torch.empty(C, device=DEV)

    def scratch(dy, x):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        pkg.liec_layer_norm_backward(dy, x, mean, rstd, dweight=dw, need_dx=False)
        torch.cuda.synchronize()
        return torch.cuda.max_memory_allocated() - before

    whole, xs, dys = scratch(dy[..., :C].contiguous(), x[..., :C].contiguous()), x[..., :C], dy[..., 3:3 + C]
    assert scratch(dys, xs) == whole
    assert scratch(dys, xs.contiguous()) == whole


def _turned(t):
    """The same values with the last but one dimension outermost in memory."""
    return t.transpose(0, t.dim() - 2).contiguous().transpose(0, t.dim() - 2)


@pytest.mark.parametrize("shape", [(6, 11, 40), (6, 11, 5), (4, 7, 17_000)])
def test_outputs_of_another_order(shape):
    say(f"case layer norm {shape}, outputs of another order than their inputs")
    x, dy, w, b = _shared(shape, seed=203)
    _forward_and_backward(x, dy, w, b, out=_turned(torch.empty_like(x)), dx=_turned(torch.empty_like(x)))
    _forward_and_backward(_turned(x), dy, w, b, out=torch.empty_like(x))
    _forward_and_backward(x, _turned(dy), w, b)


def test_rows_that_no_two_distances_describe():
    import paper_2402_11857_amd as pkg

    say("case layer norm, four dimensions in reverse")
    x, _, w, b = _shared((3, 2, 4, 130), seed=204)
    with pytest.raises(ValueError):
        pkg.liec_layer_norm(_turned(x), w, b)
    with pytest.raises(ValueError):
        pkg.liec_layer_norm(x, w, b, out=_turned(x))


def test_rows_in_two_groups_of_dimensions():
    say("case layer norm, four dimensions, the first two against the third")
    x, dy, w, b = _shared((3, 4, 5, 72), seed=205)
    wide = torch.empty(5, 3, 4, 72 + 9, dtype=x.dtype, device=DEV)
    view = wide.permute(1, 2, 0, 3)[..., 2:74]               # [3, 4, 5, 72]: the first two dimensions are one
    view.copy_(x)
    _forward_and_backward(view, dy, w, b)
    _forward_and_backward(x, dy, w, b, out=view.clone(memory_format=torch.preserve_format), dx=view)


def test_more_rows_than_one_worker_may_have():
    import paper_2402_11857_amd as pkg

    say("case layer norm, 2^31 rows of an expanded tensor, arguments only")
    shape = (2, 1 << 30, 8)                                  # nothing is asked for, so nothing is computed
    x = torch.ones(8, dtype=torch.bfloat16, device=DEV).expand(shape)
    mean = torch.empty(shape[:2], device=DEV)
    assert pkg.liec_layer_norm_backward(x, x, mean, mean, need_dx=False) is None
