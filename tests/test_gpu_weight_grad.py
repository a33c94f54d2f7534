"""Gradients of a linear layer's weight and bias from an 8-bit checkpoint of its input, against the definition in 64 bits.

Bounds: every product is exact (dy is taken apart into P = 1, 2, 3 bf16 numbers, the checkpoint's values are bf16 numbers), so what rounds is their sum: at most
P min(R, 8192) + 64 fp32 additions, each off by at most 2^-23 of the sum of magnitudes (a matrix instruction may cut off where it adds),
then fp64 and one rounding to the output's type."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _activations import activations, value  # noqa: E402
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, TINY, U, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS
PARTS = {"bf16": 1, "fp16": 2, "fp32": 3}


def _name(dtype):
    return next(k for k, v in DTYPES.items() if v == dtype)


def _inputs(N, R, O, C, dtype, seed):
    import paper_2402_11857_amd as pkg

    saved = pkg.liec_checkpoint_save(activations((N, R, C), dtype, seed))
    dy = (0.1 * torch.randn(N, R, O, generator=generator(seed + 1), device=DEV)).to(DTYPES[dtype])
    return dy, saved


def _check(dy, saved, dw, db):
    """dw [N, O, C] or [O, C]."""
    g, x = dy.double().reshape(dy.shape[0], -1, dy.shape[-1]), value(saved).reshape(dy.shape[0], -1, saved.values.shape[-1])
    if dw.dim() == 2:
        g, x = g.reshape(1, -1, g.shape[-1]), x.reshape(1, -1, x.shape[-1])
    K = PARTS[_name(dy.dtype)] * min(g.shape[1], 8192) + 64
    for i in range(g.shape[0]):
        gi, xi = g[i].t().contiguous(), x[i]
        for got, want, mass, what in ((dw, gi @ xi, gi.abs() @ xi.abs(), "dweight"), (db, gi.sum(1), gi.abs().sum(1), "dbias")):
            if got is None:
                continue
            one = got[i] if dw.dim() == 3 else got
            bound = K * 2.0 ** -23 * mass
            t = _name(got.dtype)
            if t != "fp32":
                bound = bound + 1.01 * U[t] * (want.abs() + bound)
            assert_within(one, want, bound + TINY[t], f"{what} of worker {i}")


# both sides of every change of tiles, splits and steps; lengths of no vector; one row, one column
SIZES = [(1, 1, 1, 1), (2, 1, 5, 33), (3, 2, 64, 64), (2, 7, 65, 63), (4, 32, 10, 160), (1, 63, 100, 31), (2, 64, 128, 128), (1, 65, 129, 127), (2, 300, 130, 257),
         (1, 1000, 17, 1001), (3, 129, 1, 300), (1, 257, 300, 1), (1, 8193, 40, 72), (1, 20_001, 70, 66), (5, 255, 96, 80), (1, 640, 512, 520), (2, 100, 385, 511), (70, 9, 12, 20),
         (1, 4100, 256, 264), (2, 513, 1030, 90), (1, 90, 90, 2050),
         (2, 333, 272, 304), (1, 129, 136, 144), (3, 200, 520, 400), (1, 8200, 264, 272), (2, 64, 72, 1008), (1, 1, 512, 512), (9, 65, 256, 256)]


@pytest.mark.parametrize("N,R,O,C", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_sizes_and_types(N, R, O, C, dtype):
    import paper_2402_11857_amd as pkg

    say(f"case weight gradient N={N} R={R} O={O} C={C} {dtype}")
    dy, saved = _inputs(N, R, O, C, dtype, seed=R + O + C)
    db = torch.full((N, O), 9.0, device=DEV)
    dw = pkg.liec_weight_grad(dy, saved, dbias=db)
    assert dw.shape == (N, O, C) and dw.dtype == torch.float32
    _check(dy, saved, dw, db)
    # columns of wider rows, at an odd place; nothing around them is touched; no bias
    rows = torch.full((N, O * C + O + 41), 7.0, device=DEV)
    at = rows[:, 13:13 + O * C].view(N, O, C)
    assert pkg.liec_weight_grad(dy, saved, dweight=at) is at
    assert torch.equal(at, dw) and (rows[:, :13] == 7).all() and (rows[:, 13 + O * C:] == 7).all()
    # one sum over all workers
    one, bias = torch.empty(O, C, device=DEV), torch.empty(O, device=DEV)
    pkg.liec_weight_grad(dy, saved, dweight=one, dbias=bias)
    _check(dy, saved, one, bias)


@pytest.mark.parametrize("params", list(DTYPES))
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_types_and_strides(dtype, params):
    import paper_2402_11857_amd as pkg

    say(f"case weight gradient strides {dtype} {params}")
    for N, R, O, C in ((3, 50, 40, 70), (2, 9000, 33, 17), (2, 150, 133, 144), (2, 90, 75, 80)):
        dy, saved = _inputs(N, R, O, C, dtype, seed=5)
        room = torch.full((N, O + 3, C + 5), 4.0, dtype=DTYPES[params], device=DEV)
        dw, bias = room[:, 1:1 + O, 2:2 + C], torch.full((N, O + 9), 4.0, dtype=DTYPES[params], device=DEV)
        db = bias[:, 3:3 + O]
        pkg.liec_weight_grad(dy, saved, dweight=dw, dbias=db)
        _check(dy, saved, dw, db)
        edge = room.clone()
        edge[:, 1:1 + O, 2:2 + C] = 4.0
        assert (edge == 4).all() and (bias[:, :3] == 4).all() and (bias[:, 3 + O:] == 4).all()
        # dy as columns of wider rows, rows apart, workers apart, one for all
        wide = torch.empty(N, 2 * R, O + 11, dtype=dy.dtype, device=DEV)
        view = wide[:, ::2, 5:5 + O]
        view.copy_(dy)
        assert torch.equal(pkg.liec_weight_grad(view, saved), pkg.liec_weight_grad(dy, saved))
        # rows at distances of 16 bytes that are longer than dy, or overlap
        room = torch.full((N, R, 8 * (O // 8 + 2)), float("nan"), dtype=dy.dtype, device=DEV)
        room[..., 8:8 + O] = dy
        assert torch.equal(pkg.liec_weight_grad(room[..., 8:8 + O], saved), pkg.liec_weight_grad(dy, saved))
        near = torch.randn(N, R * 16 + O, generator=generator(6), device=DEV).to(dy.dtype).as_strided((N, R, O), (R * 16 + O, 16, 1))
        assert torch.equal(pkg.liec_weight_grad(near, saved), pkg.liec_weight_grad(near.contiguous(), saved))
        same = dy[:1].expand(N, R, O)
        assert torch.equal(pkg.liec_weight_grad(same, saved), pkg.liec_weight_grad(same.contiguous(), saved))


def test_images_and_single_rows():
    import paper_2402_11857_amd as pkg

    say("case weight gradient of images and single rows")
    x = activations((3, 2, 5, 7, 48), "bf16", seed=6)
    dy = activations((3, 2, 5, 7, 24), "bf16", seed=7)
    saved = pkg.liec_checkpoint_save(x)
    dw = pkg.liec_weight_grad(dy, saved)
    _check(dy, saved, dw, None)
    one = pkg.Checkpoint(saved.values[:, 0, 0, 0].contiguous(), saved.exponents[:, 0, 0, 0].contiguous())
    dw = pkg.liec_weight_grad(dy[:, 0, 0, 0].contiguous(), one)
    assert torch.equal(dw.double(), dy[:, 0, 0, 0].double()[:, :, None] * value(one)[:, None])


def test_whole_numbers_are_exact():
    import paper_2402_11857_amd as pkg

    say("case weight gradient of whole numbers")
    gen = generator(8)
    for dtype in DTYPES:
        for N, R, O, C in ((2, 333, 75, 140), (1, 2000, 260, 300)):
            x = torch.randint(-60, 61, (N, R, C), generator=gen, device=DEV).to(DTYPES[dtype])
            x[..., ::32] = 127.0                             # every group's exponent: the integers themselves
            dy = torch.randint(-8, 9, (N, R, O), generator=gen, device=DEV).to(DTYPES[dtype])
            saved = pkg.liec_checkpoint_save(x)
            db = torch.empty(N, O, device=DEV)
            dw = pkg.liec_weight_grad(dy, saved, dbias=db)
            assert torch.equal(dw.double(), torch.stack([dy[i].double().t().contiguous() @ x[i].double() for i in range(N)]))
            assert torch.equal(db.double(), dy.double().sum(1))


def test_every_bit_of_dy_counts():
    """One row: products of single numbers, exact in 64 bits, rounded once (dy in fp32 is three bf16 numbers, whose products are added up)."""
    import paper_2402_11857_amd as pkg

    say("case weight gradient, bits of dy")
    gen = generator(9)
    saved = pkg.liec_checkpoint_save(torch.ones(1, 1, 32, device=DEV))
    for dtype, t in DTYPES.items():
        bits = torch.randint(0, 1 << (31 if dtype == "fp32" else 15), (1, 1, 4096), generator=gen, device=DEV)
        dy = (bits.to(torch.int32).view(torch.float32) if dtype == "fp32" else bits.to(torch.int16).view(t))
        dy = torch.where(torch.isfinite(dy) & ((dy.abs() > 2.0 ** -100) if dtype != "fp16" else torch.ones_like(dy, dtype=torch.bool)), dy, torch.ones_like(dy))
        dw = pkg.liec_weight_grad(dy.contiguous(), saved)
        assert torch.equal(dw[0], dy[0, 0].float()[:, None].expand(4096, 32)), dtype
        largest = torch.full((1, 1, 8), torch.finfo(t).max, dtype=t, device=DEV)
        assert torch.equal(pkg.liec_weight_grad(largest, saved)[0], largest[0, 0].float()[:, None].expand(8, 32))


def test_values_that_are_no_numbers():
    import paper_2402_11857_amd as pkg

    say("case weight gradient of infinities and NaN")
    for dtype in DTYPES:
        dy, saved = _inputs(2, 40, 20, 70, dtype, seed=10)
        clean = pkg.liec_weight_grad(dy, saved)
        for bad in (float("inf"), float("nan")):
            hit = dy.clone()
            hit[1, 7, 3] = bad
            db = torch.empty(2, 20, device=DEV)
            dw = pkg.liec_weight_grad(hit, saved, dbias=db)
            keep = torch.ones_like(dw, dtype=torch.bool)
            keep[1, 3] = False
            assert torch.equal(dw[keep], clean[keep]) and not torch.isfinite(dw[1, 3]).any() and not torch.isfinite(db[1, 3]) and torch.isfinite(db).sum() == 39
        saved.exponents[0, 5, 1] = 255
        dw = pkg.liec_weight_grad(dy, saved)
        assert torch.isnan(dw[0, :, 32:64]).all() and torch.isfinite(dw[0, :, :32]).all() and torch.isfinite(dw[0, :, 64:]).all() and torch.equal(dw[1], clean[1])


def test_no_rows():
    import paper_2402_11857_amd as pkg

    say("case weight gradient of no rows")
    saved = pkg.liec_checkpoint_save(torch.empty(3, 0, 40, device=DEV))
    dw, db = torch.full((3, 70, 40), 5.0, device=DEV), torch.full((3, 70), 5.0, device=DEV)
    pkg.liec_weight_grad(torch.empty(3, 0, 70, device=DEV), saved, dweight=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_against_differences():
    import paper_2402_11857_amd as pkg

    say("case weight gradient against differences")
    dy, saved = _inputs(2, 30, 6, 40, "fp32", seed=11)
    x = value(saved)
    dw = pkg.liec_weight_grad(dy, saved)
    # the loss is linear in the weight: a difference over any step is its gradient
    w = torch.zeros(2, 6, 40, dtype=torch.float64, device=DEV)
    for i in range(0, w.numel(), 37):
        e = w.clone()
        e.view(-1)[i] = 1.0
        y = torch.stack([x[k] @ e[k].t().contiguous() for k in range(2)])
        assert abs(float((y * dy.double()).sum()) - dw.view(-1)[i].item()) < 1e-5


def test_bits_streams_and_graphs():
    import paper_2402_11857_amd as pkg

    say("case weight gradient, bits, streams and graphs")
    for N, R, O, C in ((3, 700, 80, 96), (1, 9000, 40, 50)):
        dy, saved = _inputs(N, R, O, C, "fp16", seed=12)

        def grad():
            db = torch.empty(N, O, device=DEV)
            return pkg.liec_weight_grad(dy, saved, dbias=db), db

        want = grad()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = grad()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = grad()
        for i in range(4):
            dy.copy_(activations((N, R, O), "fp16", seed=40 + i))
            graph.replay()
            torch.cuda.synchronize()
            want = grad()
            assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_large_offsets():
    import paper_2402_11857_amd as pkg

    say("case weight gradient from 2^31 + 2^22 values of a checkpoint")
    R, C, O = 65_664, 32_768, 8
    saved = pkg.Checkpoint(torch.randint(-127, 128, (1, R, C), generator=generator(13), device=DEV, dtype=torch.int8),
                           torch.full((1, R, C // 32), 127, dtype=torch.uint8, device=DEV))
    dy = torch.zeros(1, R, O, dtype=torch.bfloat16, device=DEV)
    for o, r in enumerate((0, 1, 65_535, 65_536, 65_537, 65_600, 65_662, 65_663)):
        dy[0, r, o] = 1.0
    dw = pkg.liec_weight_grad(dy, saved)
    for o, r in enumerate((0, 1, 65_535, 65_536, 65_537, 65_600, 65_662, 65_663)):
        assert torch.equal(dw[0, o], saved.values[0, r].float())


def test_refusals():
    import paper_2402_11857_amd as pkg

    say("case weight gradient refusals")
    dy, saved = _inputs(2, 30, 8, 40, "fp32", seed=14)
    dw = torch.empty(2, 8, 40, device=DEV)
    for error, call in ((TypeError, lambda: pkg.liec_weight_grad(dy.double(), saved)), (TypeError, lambda: pkg.liec_weight_grad(dy, saved.values)),
                        (ValueError, lambda: pkg.liec_weight_grad(dy[:, :29], saved)), (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw[:1])),
                        (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw[:, :7])), (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw.transpose(1, 2))),
                        (TypeError, lambda: pkg.liec_weight_grad(dy, saved, dw, torch.empty(2, 8, device=DEV).half())),
                        (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw, torch.empty(8, device=DEV))),
                        (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw[0], torch.empty(2, 8, device=DEV))),
                        (ValueError, lambda: pkg.liec_weight_grad(dy, saved, dw, torch.empty(1, 8, device=DEV).expand(2, 8))),
                        (pkg.LiecError, lambda: pkg.liec_weight_grad(dy, saved, dw[:1].expand(2, 8, 40))), (TypeError, lambda: pkg.liec_weight_grad(dy, saved, dw.cpu())),
                        (pkg.LiecError, lambda: pkg.liec_weight_grad(dy, saved, dw, dw[:, 0, :8])), (ValueError, lambda: pkg.liec_weight_grad(dy.transpose(1, 2), saved)),
                        (TypeError, lambda: pkg.liec_weight_grad(dy, saved, None, torch.empty(2, 8, device=DEV).half()))):
        with pytest.raises(error):
            call()
    before = dw._version
    pkg.liec_weight_grad(dy, saved, dw)
    assert dw._version > before
