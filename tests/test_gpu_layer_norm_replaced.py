"""A weight gradient in the place of the weight, and refusals of memory that is shared in part."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from test_gpu_layer_norm import _inputs  # noqa: E402

pytestmark = GPU_MARKS


@pytest.mark.parametrize("C", [5, 200, 1001, 5000, 17_000])
@pytest.mark.parametrize("R", [2, 700])
def test_the_weight_is_replaced_by_its_gradient(C, R):
    import paper_2402_11857_amd as pkg

    say(f"case layer norm, weight replaced by a gradient, R={R} C={C}")
    x, dy, w, b = _inputs((3, R, C), "bf16", seed=C)
    for weight in (w, w[0].clone()):
        _, mean, rstd = pkg.liec_layer_norm(x, weight)
        dw, db = torch.empty_like(weight), torch.empty_like(weight)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, weight, dweight=dw, dbias=db)
        for k in (0, 1):
            place, other = weight.clone(), torch.empty_like(weight)
            got = pkg.liec_layer_norm_backward(dy, x, mean, rstd, place, dweight=(place, other)[k], dbias=(other, place)[k])
            assert torch.equal(got, dx) and torch.equal((place, other)[k], dw) and torch.equal((other, place)[k], db)


def test_refusals():
    import paper_2402_11857_amd as pkg

    say("case layer norm, memory shared in part")
    wide = torch.zeros(2, 6, 200, device=DEV)
    x, w = wide[..., :64], torch.ones(2, 100, device=DEV)
    for out in (wide[..., 63:127], wide[..., 1:65], wide.flatten()[4:4 + 768].view(2, 6, 64)):
        with pytest.raises(pkg.LiecError):
            pkg.liec_layer_norm(x, out=out)
    y, mean, rstd = pkg.liec_layer_norm(x, out=wide[..., 64:128])
    for bad in (dict(dweight=w[:, :64], dbias=w[:, 36:]), dict(dweight=x[:, 0])):
        with pytest.raises(pkg.LiecError):
            pkg.liec_layer_norm_backward(y, x, mean, rstd, **bad)
    assert bool((wide[..., :64] == 0).all()) and bool((w == 1).all())
