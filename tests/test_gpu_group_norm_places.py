"""Group normalisation in two passes, in the place of its operands, and its gradients beyond 2^31 values."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _activations import activations, value  # noqa: E402
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, generator  # noqa: E402
from test_gpu_group_norm import check_backward, check_forward  # noqa: E402

pytestmark = GPU_MARKS


@pytest.mark.parametrize("shape,G", [((2, 1, 4100, 64), 4), ((1, 2, 4100, 90), 9), ((2, 2, 900, 6), 3), ((1, 2, 40, 1031), 1), ((1, 1, 20_003, 41), 1)])
@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_two_passes_in_place(shape, G, act, dtype):
    """Equal bits in place of x or dy and elsewhere: contiguous, and as columns of wider rows around which nothing changes."""
    import paper_2402_11857_amd as pkg

    say(f"case two passes in place {shape} {act} {dtype}")
    N, C = shape[0], shape[-1]
    gen = generator(41)
    x, dy = activations(shape, dtype, 40), (0.1 * torch.randn(shape, generator=gen, device=DEV)).to(DTYPES[dtype])
    w, b = 1 + 0.2 * torch.randn(N, C, generator=gen, device=DEV), 0.2 * torch.randn(N, C, generator=gen, device=DEV)
    y, mean, rstd, saved = pkg.liec_group_norm(x, G, w, b, activation=act, save=True)
    check_forward(x, G, w, b, act, y, mean, rstd)
    grads = {}
    for name, at, seen in (("x", x, x), ("checkpoint", saved, value(saved))):
        dw, db = torch.empty_like(w), torch.empty_like(w)
        dx = pkg.liec_group_norm_backward(dy, at, mean, rstd, w, b, activation=act, dweight=dw, dbias=db)
        check_backward(dy, seen, mean, rstd, G, w, b, act, dx, dw, db)
        grads[name] = dx, dw, db

    def plain(t):
        return t.clone(), None

    def wide(t):
        room = torch.full((*shape[:-1], C + 13), 3.0, dtype=t.dtype, device=DEV)
        room[..., 5:5 + C] = t
        return room[..., 5:5 + C], room

    for place in (plain, wide):
        here, room = place(x)
        out, m, r, kept = pkg.liec_group_norm(here, G, w, b, activation=act, out=here, save=True)
        assert out is here and torch.equal(here, y) and torch.equal(m, mean) and torch.equal(r, rstd)
        assert torch.equal(kept.values, saved.values) and torch.equal(kept.exponents, saved.exponents)
        for name, given in (("x", "x"), ("x", "dy"), ("checkpoint", "dy")):
            (here, room), (grad, other) = place(x), place(dy)
            dw, db = torch.empty_like(w), torch.empty_like(w)
            into, rest = (here, room) if given == "x" else (grad, other)
            pkg.liec_group_norm_backward(grad, saved if name == "checkpoint" else here, mean, rstd, w, b, activation=act, dx=into, dweight=dw, dbias=db)
            assert all(torch.equal(p, q) for p, q in zip((into, dw, db), grads[name])), (name, given)
            if rest is not None:
                assert (rest[..., :5] == 3).all() and (rest[..., 5 + C:] == 3).all()


def test_gradients_beyond_2_31_values():
    import paper_2402_11857_amd as pkg

    say("case group norm gradients of 2^31 + 2^21 values")
    N, B, S, C, G = 2, 1, 32_800, 32_768, 8
    gen = generator(42)
    x = torch.empty(N, B, S, C, dtype=torch.bfloat16, device=DEV).normal_(0.5, 1.0, generator=gen)
    dy = torch.empty(N, B, S, C, dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.1, generator=gen)
    w, b = 1 + 0.2 * torch.randn(N, C, generator=gen, device=DEV), 0.2 * torch.randn(N, C, generator=gen, device=DEV)
    _, mean, rstd, saved = pkg.liec_group_norm(x, G, w, b, activation="silu", save=True)
    dx = torch.empty_like(x)
    for kept in (x, saved):
        dw, db = torch.empty_like(w), torch.empty_like(w)
        pkg.liec_group_norm_backward(dy, kept, mean, rstd, w, b, activation="silu", dx=dx, dweight=dw, dbias=db)
        for g in (0, G - 1):
            cut = slice(g * 4096, (g + 1) * 4096)
            at = x[1:, :, :, cut] if kept is x else value((saved.values[1:, :, :, cut], saved.exponents[1:, :, :, g * 128:(g + 1) * 128]))
            stats = (t[1:, :, g:g + 1].contiguous() for t in (mean, rstd))
            check_backward(dy[1:, :, :, cut], at, *stats, 1, w[1:, cut], b[1:, cut], "silu", dx[1:, :, :, cut], dw[1:, cut], db[1:, cut])
            del at
