"""SiLU behind a group normalisation, and its gradients, far below zero."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, TINY, U, U32, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS
EPS = 1e-5
# images that a block holds, images in two passes, channels fewer than a vector
PATHS = [((2, 2, 24, 64), 4), ((2, 1, 5000, 64), 4), ((1, 2, 300, 6), 3)]


def _images(shape, dtype, seed):
    gen = generator(seed)
    x, dy = (torch.randn(shape, generator=gen, device=DEV).to(DTYPES[dtype]) for _ in range(2))
    return x, dy


@pytest.mark.parametrize("shape,G", PATHS)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_silu_far_below_zero_is_zero(shape, G, dtype):
    """With weights of zero z is the bias.  Against z / (1 + exp(-z)) in 64 bits: the exponential is off by |z| u (16-bit results) or
    a few u, the sum, the reciprocal and the product by a few u more; a reciprocal under 2^-126 may come as 0, which is off by
    |z| 2^-126 at most, and by nothing where |z| > 104: there the result is under the smallest number."""
    import paper_2402_11857_amd as pkg

    say(f"case SiLU far below zero {shape} {dtype}")
    x, dy = _images(shape, dtype, seed=1)
    N, C = shape[0], shape[-1]
    values = torch.tensor([-1.0, -50.0, -85.0, -87.0, -88.0, -89.0, -100.0, -104.0, -1e3, -1e10, -1e30, -1e36, -1e38, -3e38, 0.0, 88.0], device=DEV)
    b = values.repeat(-(-N * C // 16))[:N * C].view(N, C).contiguous()
    y, mean, rstd = pkg.liec_group_norm(x, G, torch.zeros_like(b), b, EPS, activation="silu")
    z = b.double()[:, None, None].expand(shape)
    want = z * torch.sigmoid(z)
    bound = (16 + (z.abs() if dtype != "fp32" else 0.0)) * U32 * want.abs() + z.abs().clamp(max=104.0) * 2.0 ** -126
    if dtype != "fp32":
        bound = bound + 1.01 * U[dtype] * (want.abs() + bound)
    keep = want.abs() <= torch.finfo(DTYPES[dtype]).max
    assert_within(y[keep], want[keep], bound[keep] + TINY[dtype], "y")
    # gradients: no slope is left from -1e3 on, whatever the value is
    far = torch.tensor([-1e3, -1e30, -1e36, -1e38, -3e38], device=DEV).repeat(-(-N * C // 5))[:N * C].view(N, C).contiguous()
    w = torch.ones_like(far)
    y, mean, rstd, saved = pkg.liec_group_norm(x, G, w, far, EPS, activation="silu", save=True)
    assert float(y.abs().max()) <= 1e-30
    for at in (x, saved):
        dw, db = torch.full_like(w, 9.0), torch.full_like(w, 9.0)
        dx = pkg.liec_group_norm_backward(dy, at, mean, rstd, w, far, activation="silu", dweight=dw, dbias=db)
        for t in (dx, dw, db):
            assert float(t.abs().max()) <= 1e-30
