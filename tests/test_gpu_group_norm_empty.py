"""Statistics of images without positions."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402

pytestmark = GPU_MARKS


def test_images_without_positions_have_no_mean():
    import paper_2402_11857_amd as pkg

    say("case statistics of images without positions")
    for shape in ((2, 3, 0, 16), (2, 3, 4, 0, 16), (1, 50_000, 0, 64)):
        for save in (False, True):
            # what was there before, if the memory is used again
            torch.full((shape[0] * shape[1] * 4,), 7.0, device=DEV)
            y, mean, rstd, *saved = pkg.liec_group_norm(torch.empty(shape, device=DEV), 4, save=save)
            assert y.shape == shape and mean.shape == rstd.shape == (shape[0], shape[1], 4)
            assert torch.isnan(mean).all() and torch.isnan(rstd).all()
    _, mean, rstd = pkg.liec_group_norm(torch.empty(2, 0, 5, 16, device=DEV), 4)
    assert mean.shape == rstd.shape == (2, 0, 4)
