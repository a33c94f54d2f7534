"""Bias gradients of many rows: fp32 chains of at most 256 rows; and weight gradients from tiles at 16-byte distances beyond 2^31 values."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, U32, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS


def _saved(N, R, C):
    import paper_2402_11857_amd as pkg

    return pkg.Checkpoint(torch.zeros(N, R, C, dtype=torch.int8, device=DEV), torch.full((N, R, -(-C // 32)), 127, dtype=torch.uint8, device=DEV))


# enough tiles that the rows are not split: 256 x 256, 128 x 128 and 64 x 64 values, at 16-byte distances and not; and splits of more rows
SIZES = [(256, 131_072), (128, 65_536), (255, 130_817), (127, 65_409), (264, 33_000), (64, 32_768), (40, 32_600)]


@pytest.mark.parametrize("O,C", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("R", [8192, 20_000])
def test_rows_of_one_sign(O, C, dtype, R):
    """Rows whose last bits get lost in long chains.  The sums of a chain of 256 additions grow evenly to s; additions whose result lies in
    [2^e, 2^(e + 1)) are off by 2^(e - 24) at most, half of them in the highest such range: (1 + 1/4 + 1/16 + ...) 128 u s,
    at most 256 u s / 3 * (s against 2^(e + 1): 1 at most) < 86 u s.  What a block and the splits add to them takes less than 10 u."""
    import paper_2402_11857_amd as pkg

    say(f"case bias gradient O={O} C={C} R={R} {dtype}")
    saved = _saved(1, R, C)
    for bit in (-14, -15, -16):
        small = torch.tensor(0.9 * 2.0 ** bit, device=DEV)
        if dtype == "fp32":
            dy = (1.0 + small).expand(1, R, O).contiguous()
        else:                                                # rows of 1 and of what a long sum loses, in turn
            dy = torch.ones(1, R, O, device=DEV)
            dy[:, ::2] = small
            dy = dy.to(DTYPES[dtype])
        db = torch.empty(1, O, device=DEV)
        dw = pkg.liec_weight_grad(dy, saved, dbias=db)
        assert not dw.any()
        want = dy.double().sum(1)
        assert_within(db, want, 96 * U32 * want, f"dbias, 2^{bit}")


def _few_rows(R):
    return [0, 1, 63, 64, R // 2, R - 65, R - 2, R - 1]


def test_aligned_checkpoint_beyond_2_31_values():
    import paper_2402_11857_amd as pkg

    R, C, O = 65_664, 32_768, 256
    say("case weight gradient, tiles from 2^31 + 2^22 values of a checkpoint")
    saved = pkg.Checkpoint(torch.randint(-127, 128, (1, R, C), generator=generator(13), device=DEV, dtype=torch.int8),
                           torch.full((1, R, C // 32), 127, dtype=torch.uint8, device=DEV))
    for dtype in DTYPES.values():
        dy = torch.zeros(1, R, O, dtype=dtype, device=DEV)
        for o, r in enumerate(_few_rows(R)):
            dy[0, r, o] = 1.0
        dw = pkg.liec_weight_grad(dy, saved)
        for o, r in enumerate(_few_rows(R)):
            assert torch.equal(dw[0, o], saved.values[0, r].float())
        assert not dw[0, 8:].any()


def test_aligned_rows_beyond_2_31_values():
    import paper_2402_11857_amd as pkg

    R, C, O, apart = 4100, 272, 264, 1 << 20
    say("case weight gradient, tiles from rows 2^20 values apart")
    saved = pkg.liec_checkpoint_save(torch.randn(2, R, C, generator=generator(14), device=DEV))
    room = torch.empty(2 * R * apart, dtype=torch.bfloat16, device=DEV)
    dy = room.as_strided((2, R, O), (R * apart, apart, 1))
    dy.copy_(torch.randn(2, R, O, generator=generator(15), device=DEV))
    db, same = torch.empty(2, O, device=DEV), torch.empty(2, O, device=DEV)
    dw = pkg.liec_weight_grad(dy, saved, dbias=db)
    assert torch.equal(dw, pkg.liec_weight_grad(dy.contiguous(), saved, dbias=same)) and torch.equal(db, same)


def test_weights_beyond_2_31_values():
    import paper_2402_11857_amd as pkg

    R, O, C = 16, 66_000, 32_768
    say("case weight gradient of 2^31 + 2^23 weights")
    saved = pkg.Checkpoint(torch.randint(-127, 128, (1, R, C), generator=generator(16), device=DEV, dtype=torch.int8),
                           torch.full((1, R, C // 32), 127, dtype=torch.uint8, device=DEV))
    dy = torch.randint(-8, 9, (1, R, O), generator=generator(17), device=DEV).to(torch.bfloat16)
    dw = pkg.liec_weight_grad(dy, saved)
    for o in (0, 255, 256, 65_535, 65_536, O - 65, O - 1):
        assert torch.equal(dw[0, o].double(), (dy[0, :, o].double()[:, None] * saved.values[0].double()).sum(0))
