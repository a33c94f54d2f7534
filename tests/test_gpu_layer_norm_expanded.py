"""Weight gradients of all workers in the memory of one."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from test_gpu_layer_norm import _check_backward, _check_forward, EPS, _inputs  # noqa: E402

pytestmark = GPU_MARKS


def test_expanded_gradients_are_refused():
    import paper_2402_11857_amd as pkg

    say("case layer norm, expanded weight gradients")
    x, dy, w, b = _inputs((3, 4, 64), "fp32", seed=207)
    y, mean, rstd = pkg.liec_layer_norm(x, w, b)
    for bad in (dict(dweight=torch.zeros(64, device=DEV).expand(3, 64)), dict(dbias=torch.zeros(64, device=DEV).expand(3, 64)),
                dict(dweight=torch.zeros(64, device=DEV).expand(3, 64), dbias=torch.zeros(64, device=DEV).expand(3, 64))):
        with pytest.raises(ValueError):                      # one vector cannot hold each worker's own sum
            pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, **bad)
        assert all(bool((t == 0).all()) for t in bad.values())
    # expanded weights are only read, and one worker's gradient has no distance to the next
    _check_forward(x, w[0].expand(3, 64), None, EPS, *pkg.liec_layer_norm(x, w[0].expand(3, 64), eps=EPS))
    one = torch.zeros(64, device=DEV).expand(1, 64)
    dx = pkg.liec_layer_norm_backward(dy[:1], x[:1], mean[:1], rstd[:1], w[:1], dweight=one)
    _check_backward(dy[:1], x[:1], mean[:1], rstd[:1], w[:1], dx, one, None)
