"""Group normalisation with an activation, channels last, and its gradients against the definitions in 64 bits.

Bounds, with u = 2^-24 and chains of at most K = min(S, 256) + 40 fp32 additions per channel (a thread's positions, 6 steps inside a
wave, a block's waves; groups are put together in fp64): values are added up around a value p of the group, so the mean is off by at most K u D with D = max |x - p|
<= 2 max |x - mu|, plus u |mu|, and the variance by K u times the mean of (x - p)^2, which is at most var + D^2.  Products, shifts and the activation
add a few u; an activation passes errors on by at most its slope, 1 (ReLU) or 1.1 (SiLU), whose own slope is at most 1/2.  The result
is rounded once to its type."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _activations import activations, expected_checkpoint, value  # noqa: E402
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, TINY, U, U32, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS
EPS = 1e-5
ACTS = ("none", "relu", "silu")


def _name(dtype):
    return next(k for k, v in DTYPES.items() if v == dtype)


def _inputs(shape, dtype, seed, params="fp32", offset=0.5):
    gen = generator(seed + 1000)
    N, C = shape[0], shape[-1]
    x = activations(shape, dtype, seed, offset)
    dy = (torch.randn(shape, generator=gen, device=DEV) * 0.1).to(DTYPES[dtype])
    w = (1 + 0.2 * torch.randn(N, C, generator=gen, device=DEV)).to(DTYPES[params])
    b = (0.2 * torch.randn(N, C, generator=gen, device=DEV)).to(DTYPES[params])
    return x, dy, w, b


def _five(t, G):
    """[N, B, ..., C] as [N, B, S, G, C / G]."""
    return t.reshape(t.shape[0], t.shape[1], -1, G, t.shape[-1] // G)


def _param(p, G, fill):
    """[C] or [N, C] in 64 bits, to go with that."""
    if p is None:
        return torch.full((), fill, dtype=torch.float64, device=DEV)
    p = p.double()
    return p.reshape(-1, 1, 1, G, p.shape[-1] // G)


def _round(bound, want, t):
    if t != "fp32":
        bound = bound + 1.01 * U[t] * (want.abs() + bound)
    return bound + TINY[t]


def check_forward(x, G, w, b, act, y, mean, rstd, eps=EPS):
    v = _five(x.double(), G)
    K = min(v.shape[2], 256) + 40
    mu = v.mean((2, 4), keepdim=True)
    var = (v - mu).square().mean((2, 4), keepdim=True)
    rs = 1 / torch.sqrt(var + eps)
    D = 2 * (v - mu).abs().amax((2, 4), keepdim=True)
    off_mu = (K * D + 2 * mu.abs()) * U32
    off_var = 1.01 * K * U32 * (var + D ** 2) + 2 * U32 * eps
    off_rs = rs * (0.5 * off_var / (var + eps) * 1.1 + 2 * U32)
    assert mean.dtype == rstd.dtype == torch.float32
    assert_within(mean, mu[:, :, 0, :, 0], off_mu[:, :, 0, :, 0] + 1e-45, "mean")
    assert_within(rstd, rs[:, :, 0, :, 0], off_rs[:, :, 0, :, 0], "rstd")
    wd, bd = _param(w, G, 1.0), _param(b, G, 0.0)
    h = (v - mu) * rs
    z = h * wd + bd
    off_z = wd.abs() * (off_mu * rs + h.abs() * (off_rs / rs + 4 * U32)) * 1.01 + 2 * U32 * z.abs()
    want = z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z
    bound = 1.1 * off_z + 10 * U32 * want.abs()
    assert_within(y.reshape(v.shape), want, _round(bound, want, _name(x.dtype)), "y")


def check_backward(dy, x, mean, rstd, G, w, b, act, dx, dw, db):
    """x: what the gradients are taken at (of a checkpoint: what it stands for)."""
    v, g = _five(x.double(), G), _five(dy.double(), G)
    K = min(v.shape[2], 256) + 40
    mu, rs = mean.double()[:, :, None, :, None], rstd.double()[:, :, None, :, None]
    wd, bd = _param(w, G, 1.0), _param(b, G, 0.0)
    h = (v - mu) * rs
    z = h * wd + bd
    off_z = 2.1 * U32 * (h * wd).abs() + U32 * z.abs()
    if act == "relu":
        dz, off = torch.where(z > 0, g, torch.zeros_like(g)), torch.zeros_like(g)
    elif act == "silu":
        p = torch.sigmoid(z)
        dz = g * p * (1 + z * (1 - p))
        off = g.abs() * (0.5 * off_z + 12 * U32 * p * (1 + (z * (1 - p)).abs())) + U32 * dz.abs()
    else:
        dz, off = g, torch.zeros_like(g)
    a, off_a = dz * wd, (off + U32 * dz.abs()) * wd.abs()
    t = _name(dy.dtype)
    if dx is not None:
        m1, m2 = a.mean((2, 4), keepdim=True), (a * h).mean((2, 4), keepdim=True)
        off_1 = (off_a + K * U32 * a.abs()).mean((2, 4), keepdim=True)
        off_2 = (off_a * h.abs() + (K + 3) * U32 * (a * h).abs()).mean((2, 4), keepdim=True)
        want = rs * (a - m1 - h * m2)
        bound = rs * (1.01 * (off_a + off_1 + h.abs() * off_2) + 6 * U32 * (a.abs() + m1.abs() + (h * m2).abs()))
        assert_within(dx.reshape(v.shape), want, _round(bound, want, t), "dx")
    N, C = v.shape[0], x.shape[-1]
    for got, term, err, what in ((dw, dz * h, off * h.abs() + 3 * U32 * (dz * h).abs(), "dweight"), (db, dz, off, "dbias")):
        if got is None:
            continue
        over = (1, 2) if got.dim() == 2 else (0, 1, 2)
        want, mass, err = term.sum(over).reshape(got.shape), term.abs().sum(over).reshape(got.shape), err.sum(over).reshape(got.shape)
        assert_within(got, want, _round(1.01 * (err + K * U32 * mass), want, _name(got.dtype)), what)


def run_both(x, dy, G, w, b, act, eps=EPS):
    """Forward with and without a checkpoint, backward from x and from the checkpoint, everything checked."""
    import paper_2402_11857_amd as pkg

    y, mean, rstd = pkg.liec_group_norm(x, G, w, b, eps, activation=act)
    check_forward(x, G, w, b, act, y, mean, rstd, eps)
    again, mean2, rstd2, saved = pkg.liec_group_norm(x, G, w, b, eps, activation=act, save=True)
    assert torch.equal(again, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    q, s = expected_checkpoint(x)
    assert torch.equal(saved.values, q) and torch.equal(saved.exponents, s)
    for kept, at in ((x, x), (saved, value(saved))):
        dw, db = (None if p is None else torch.full_like(p, 9.0) for p in (w, b))
        dx = pkg.liec_group_norm_backward(dy, kept, mean, rstd, w, b, activation=act, dweight=dw, dbias=db)
        check_backward(dy, at, mean, rstd, G, w, b, act, dx, dw, db)


# positions below, at and above what a thread, a block and a chain take; channels shorter than a vector, odd, in one and many tiles
SHAPES = [((1, 1, 1, 1), 1), ((2, 1, 1, 4), 2), ((3, 2, 5, 7), 7), ((1, 3, 9, 8), 1), ((2, 2, 4, 9), 3), ((2, 3, 17, 24), 3), ((1, 2, 64, 30), 3), ((3, 2, 33, 33), 11),
          ((2, 2, 49, 64), 8), ((5, 3, 27 * 31, 90), 9), ((1, 1, 3000, 8), 2), ((1, 2, 700, 256), 32), ((2, 1, 130, 513), 1), ((1, 2, 50, 1030), 5), ((2, 1, 7, 4096), 64),
          ((1, 1, 1, 2048), 16), ((2, 40, 1, 96), 4), ((1, 300, 4, 32), 8), ((1, 1, 70_001, 3), 1), ((1, 1, 20_003, 40), 5), ((2, 2, 1025, 128), 1), ((1, 2, 2049, 16), 16),
          ((1, 1, 5000, 520), 8), ((1, 1, 257, 4097), 17), ((3, 1, 300, 65), 65),
          ((2, 2, 30, 512), 1), ((1, 3, 20, 1024), 2), ((2, 4, 3, 416), 1), ((3, 6, 9, 72), 1), ((2, 3, 100, 44), 11), ((1, 2, 700, 44), 11), ((4, 16, 1, 1000), 8),
          ((2, 2, 513, 200), 25), ((2, 32, 2, 40), 5), ((1, 64, 1, 16), 1), ((2, 5, 1, 8), 8), ((1, 2, 4096, 64), 2), ((1, 2, 4097, 64), 2), ((2, 2, 1023, 96), 3)]


@pytest.mark.parametrize("shape,G", SHAPES)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_shapes_and_types(shape, G, dtype):
    say(f"case group norm {shape} G={G} {dtype}")
    for act in ACTS:
        run_both(*_inputs(shape, dtype, seed=sum(shape) + G)[:2], G, *_inputs(shape, dtype, seed=sum(shape) + G)[2:], act)


@pytest.mark.parametrize("params", list(DTYPES))
def test_types_and_forms_of_parameters(params):
    import paper_2402_11857_amd as pkg

    say(f"case group norm, parameters {params}")
    x, dy, w, b = _inputs((3, 2, 6, 5, 48), "bf16", seed=2, params=params)
    run_both(x, dy, 6, w, b, "silu")
    run_both(x, dy, 6, w[0], b[0], "relu")                  # one vector for all workers
    run_both(x, dy, 6, w, None, "relu")
    run_both(x, dy, 6, None, b, "silu")
    run_both(x, dy, 6, None, None, "none")
    run_both(x, dy, 6, w[:1].expand(3, 48)[1], b[1], "none")
    # sums over all workers under weights of each, columns of rows as weights and for their gradients
    y, mean, rstd = pkg.liec_group_norm(x, 6, w, b, activation="silu")
    dw, db = torch.empty(48, dtype=w.dtype, device=DEV), torch.empty(48, dtype=w.dtype, device=DEV)
    dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="silu", dweight=dw, dbias=db)
    check_backward(dy, x, mean, rstd, 6, w, b, "silu", dx, dw, db)
    rows, grads = torch.full((3, 131), 7.0, dtype=w.dtype, device=DEV), torch.full((3, 131), 7.0, dtype=w.dtype, device=DEV)
    rows[:, 5:53], rows[:, 53:101] = w, b
    assert torch.equal(pkg.liec_group_norm(x, 6, rows[:, 5:53], rows[:, 53:101], activation="silu")[0], y)
    pkg.liec_group_norm_backward(dy, x, mean, rstd, rows[:, 5:53], rows[:, 53:101], activation="silu", dweight=grads[:, 5:53], dbias=grads[:, 53:101])
    check_backward(dy, x, mean, rstd, 6, w, b, "silu", None, grads[:, 5:53], grads[:, 53:101])
    assert (grads[:, :5] == 7).all() and (grads[:, 101:] == 7).all()
    # only some of the gradients
    only = torch.empty_like(w)
    assert pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="silu", dbias=only, need_dx=False) is None
    assert torch.equal(only, grads[:, 53:101])
    assert torch.equal(pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="silu"), dx)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_strides_and_places(dtype):
    import paper_2402_11857_amd as pkg

    say(f"case group norm strides {dtype}")
    base, grad, w, b = _inputs((4, 5, 6, 7, 64), dtype, seed=4)
    for cut in (lambda t: t[..., 8:40], lambda t: t[..., 3:36], lambda t: t[:, :, :4], lambda t: t[:, 1:3, :, :, :32], lambda t: t[::2, :, 1:2, :, 5:14], lambda t: t[:, ::2, :, 2:3],
                lambda t: t[:, :, ::2, :4][:, :, :, 0:1, 1:], lambda t: t.flip(1)[..., :16], lambda t: t[:1].expand(4, 5, 6, 7, 64)):
        x, dy = cut(base), cut(grad)
        C, N = x.shape[-1], x.shape[0]
        G = next(g for g in (4, 3, 1) if C % g == 0)
        wi, bi = w[:N, :C].contiguous(), b[:N, :C].contiguous()
        y, mean, rstd = pkg.liec_group_norm(x, G, wi, bi, activation="silu")
        check_forward(x.contiguous(), G, wi, bi, "silu", y, mean, rstd)
        dw, db = torch.empty_like(wi), torch.empty_like(bi)
        dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, wi, bi, activation="silu", dweight=dw, dbias=db)
        check_backward(dy.contiguous(), x.contiguous(), mean, rstd, G, wi, bi, "silu", dx, dw, db)
        saved = pkg.liec_group_norm(x, G, wi, bi, activation="silu", save=True)[3]
        assert torch.equal(saved.values, expected_checkpoint(x.contiguous())[0])
        # into strided memory, and in place
        room = torch.full((*x.shape[:-1], C + 9), 3.0, dtype=x.dtype, device=DEV)
        out = room[..., 4:4 + C]
        assert pkg.liec_group_norm(x, G, wi, bi, activation="silu", out=out)[0] is out
        assert torch.equal(out, y) and (room[..., :4] == 3).all() and (room[..., 4 + C:] == 3).all()
        assert pkg.liec_group_norm_backward(dy, x, mean, rstd, wi, bi, activation="silu", dx=out) is out
        assert torch.equal(out, dx) and (room[..., :4] == 3).all() and (room[..., 4 + C:] == 3).all()
        if 0 not in x.stride():
            for given in ("x", "dy"):
                here, other = room.clone()[..., 4:4 + C], room.clone()[..., 4:4 + C]
                here.copy_(x)
                other.copy_(dy)
                assert torch.equal(pkg.liec_group_norm_backward(other, here, mean, rstd, wi, bi, activation="silu", dx=here if given == "x" else other), dx)
            here.copy_(x)
            y2, mean2, _, kept = pkg.liec_group_norm(here, G, wi, bi, activation="silu", out=here, save=True)
            assert y2 is here and torch.equal(here, y) and torch.equal(mean2, mean) and torch.equal(kept.values, saved.values)
            other.copy_(dy)
            got = pkg.liec_group_norm_backward(other, saved, mean, rstd, wi, bi, activation="silu", dx=other)
            assert torch.equal(got, pkg.liec_group_norm_backward(dy, saved, mean, rstd, wi, bi, activation="silu"))


def test_offsets_and_constants():
    import paper_2402_11857_amd as pkg

    say("case group norm, large offsets and constant groups")
    for offset in (100.0, 1e4):
        x, dy, w, b = _inputs((2, 2, 500, 32), "fp32", seed=6, offset=0.0)
        x = x + offset
        run_both(x, dy, 4, w, b, "none")
    x = torch.full((2, 3, 40, 24), 7.25, device=DEV)
    y, mean, rstd = pkg.liec_group_norm(x, 3, None, w[:, :24].contiguous())
    assert torch.equal(mean, torch.full_like(mean, 7.25)) and (rstd.double() * EPS ** 0.5 - 1).abs().max() < 4 * U32
    assert torch.equal(y, w[:, None, None, :24].expand_as(y))
    # a first position far from all others: what channels are added up around is one of them
    x, dy, w, b = _inputs((1, 1, 1000, 16), "fp32", seed=7)
    x[:, :, :4] += 1000.0
    run_both(x, dy, 2, w, b, "silu")
    # a step in the middle
    x[:, :, 500:] += 1e4
    run_both(x, dy, 2, w, b, "silu")
    # zero variance and no epsilon: an infinity times zero
    y, _, rstd = pkg.liec_group_norm(torch.ones(1, 1, 4, 8, device=DEV), 2, eps=0.0)
    assert torch.isinf(rstd).all() and torch.isnan(y).all()


def test_relu_decides_next_to_zero_in_64_bits():
    import paper_2402_11857_amd as pkg

    say("case group norm, ReLU next to zero")
    N, B, S, C, G = 2, 3, 50, 64, 4
    x, dy, w, _ = _inputs((N, B, S, C), "fp32", seed=9)
    _, mean, rstd = pkg.liec_group_norm(x, G)
    # biases that put one position of every channel next to zero: (x - mean) rstd w + b within a few units of it
    h = (_five(x.double(), G) - mean.double()[:, :, None, :, None]) * rstd.double()[:, :, None, :, None]
    h = h.reshape(N, B, S, C)
    b = -(h[:, 1, 17] * w.double()).float()
    dw, db = torch.empty_like(w), torch.empty_like(w)
    dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="relu", dweight=dw, dbias=db)
    z = h * w.double()[:, None, None] + b.double()[:, None, None]
    near = z.abs() < 4 * U32 * b.double().abs()[:, None, None]
    assert near.sum() >= N * C and (z[near] > 0).any() and (z[near] < 0).any()
    check_backward(dy, x, mean, rstd, G, w, b, "relu", dx, dw, db)
    # exactly zero: no gradient
    zero = torch.zeros_like(w)
    db.fill_(5.0)
    pkg.liec_group_norm_backward(dy, x, mean, rstd, zero, zero, activation="relu", dbias=db, need_dx=False)
    assert not db.any()


def test_silu_far_from_zero():
    import paper_2402_11857_amd as pkg

    say("case group norm, SiLU far from zero")
    x, dy, w, b = _inputs((2, 1, 64, 32), "fp32", seed=10)
    b = torch.linspace(-120.0, 120.0, 64, device=DEV).view(2, 32)
    y, mean, rstd = pkg.liec_group_norm(x, 4, w, b, activation="silu")
    check_forward(x, 4, w, b, "silu", y, mean, rstd)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="silu", dweight=dw, dbias=db)
    # beyond 87 the exponential is held at 2^126, a slope of under 1e-36 that no bound here counts
    assert torch.isfinite(dx).all() and torch.isfinite(y).all()
    keep = b > -80
    want_w, want_b = torch.zeros_like(w, dtype=torch.float64), torch.zeros_like(w, dtype=torch.float64)
    h = ((_five(x.double(), 4) - mean.double()[:, :, None, :, None]) * rstd.double()[:, :, None, :, None]).reshape(x.shape)
    z = h * w.double()[:, None, None] + b.double()[:, None, None]
    p = torch.sigmoid(z)
    dz = dy.double() * p * (1 + z * (1 - p))
    want_w, want_b = (dz * h).sum((1, 2)), dz.sum((1, 2))
    off = dy.double().abs() * (0.5 * (3.2 * U32 * z.abs() + 3 * U32 * b.double().abs()[:, None, None]) + 12 * U32 * p * (1 + (z * (1 - p)).abs()))
    assert_within(db[keep], want_b[keep], ((off + 104 * U32 * dz.abs()).sum((1, 2)))[keep] + 1e-37, "dbias")
    assert_within(dw[keep], want_w[keep], ((off * h.abs() + 108 * U32 * (dz * h).abs()).sum((1, 2)))[keep] + 1e-37, "dweight")


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_groups_with_values_that_are_no_numbers(bad):
    import paper_2402_11857_amd as pkg

    say(f"case group norm with {bad}")
    x, dy, w, b = _inputs((2, 2, 60, 48), "fp32", seed=12)
    y0, mean0, rstd0 = pkg.liec_group_norm(x, 4, w, b, activation="silu")
    dx0 = pkg.liec_group_norm_backward(dy, x, mean0, rstd0, w, b, activation="silu")
    x[1, 0, 33, 13] = bad                                    # group 1 of image (1, 0)
    y, mean, rstd, saved = pkg.liec_group_norm(x, 4, w, b, activation="silu", save=True)
    hit = torch.zeros(2, 2, 4, dtype=torch.bool, device=DEV)
    hit[1, 0, 1] = True
    wide = hit[:, :, None].repeat_interleave(12, -1).expand_as(x)
    assert torch.isnan(y[wide]).all() and torch.equal(y[~wide], y0[~wide])
    assert torch.isnan(rstd[hit]).all() and torch.equal(rstd[~hit], rstd0[~hit]) and torch.equal(mean[~hit], mean0[~hit])
    dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    assert torch.isnan(dx[wide]).all() and torch.equal(dx[~wide], dx0[~wide])
    dx = pkg.liec_group_norm_backward(dy, saved, mean, rstd, w, b, activation="silu")
    assert torch.isnan(dx[wide]).all() and saved.exponents[1, 0, 33, 0] == 255
    for place in ((0, 1, 5, 47),):                           # a gradient that is none
        dy2 = dy.clone()
        dy2[place] = bad
        dx = pkg.liec_group_norm_backward(dy2, activations((2, 2, 60, 48), "fp32", 12), mean0, rstd0, w, b, activation="none")
        assert not torch.isfinite(dx[0, 1, :, 36:]).any() and torch.isfinite(dx[0, 1, :, :36]).all() and torch.isfinite(dx[1]).all()


def test_nothing_in_an_image():
    import paper_2402_11857_amd as pkg

    say("case group norm of nothing")
    w = torch.ones(2, 16, device=DEV)
    for shape in ((2, 0, 5, 16), (2, 3, 0, 16), (2, 3, 4, 0, 16)):
        x = torch.empty(shape, device=DEV)
        y, mean, rstd, saved = pkg.liec_group_norm(x, 4, w, w, save=True)
        assert y.shape == x.shape and mean.shape == (2, shape[1], 4) and saved.values.shape == x.shape
        for out in (torch.full((2, 16), 5.0, device=DEV), torch.full((16,), 5.0, device=DEV)):
            other = torch.full_like(out, 5.0)
            dx = pkg.liec_group_norm_backward(x, saved, mean, rstd, w, w, dweight=out, dbias=other)
            assert dx.shape == x.shape and not out.any() and not other.any()


def test_gradients_against_differences():
    import paper_2402_11857_amd as pkg

    say("case group norm gradients against differences")
    for act in ("none", "silu"):
        x, dy, w, b = _inputs((2, 2, 9, 12), "fp32", seed=14)

        def loss(x, w, b):
            v = _five(x, 3)
            mu = v.mean((2, 4), keepdim=True)
            z = ((v - mu) / torch.sqrt((v - mu).square().mean((2, 4), keepdim=True) + EPS)).reshape(x.shape) * w[:, None, None] + b[:, None, None]
            return float(((z * torch.sigmoid(z) if act == "silu" else z) * dy.double()).sum())

        _, mean, rstd = pkg.liec_group_norm(x, 3, w, b, activation=act)
        dw, db = torch.empty_like(w), torch.empty_like(b)
        dx = pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, activation=act, dweight=dw, dbias=db)
        xd, wd, bd = x.double(), w.double(), b.double()
        step = 1e-5                                          # differences are off by about step^2 times third derivatives, and 1e-16 / step
        for t, got in ((xd, dx), (wd, dw), (bd, db)):
            size = float(got.abs().max())
            for i in range(0, t.numel(), max(1, t.numel() // 24)):
                old = t.view(-1)[i].item()
                t.view(-1)[i] = old + step
                up = loss(xd, wd, bd)
                t.view(-1)[i] = old - step
                down = loss(xd, wd, bd)
                t.view(-1)[i] = old
                assert abs((up - down) / (2 * step) - got.view(-1)[i].item()) <= 2e-5 * size + 1e-8


def test_equal_calls_give_equal_bits_and_images_stand_alone():
    import paper_2402_11857_amd as pkg

    say("case group norm, bits")
    for shape, G in (((4, 3, 200, 96), 8), ((2, 2, 3136, 64), 8), ((3, 5, 7, 40), 5)):
        x, dy, w, b = _inputs(shape, "bf16", seed=15)
        runs = []
        for _ in range(2):
            y, mean, rstd, saved = pkg.liec_group_norm(x, G, w, b, activation="silu", save=True)
            dw, db = torch.empty_like(w), torch.empty_like(b)
            dx = pkg.liec_group_norm_backward(dy, saved, mean, rstd, w, b, activation="silu", dweight=dw, dbias=db)
            runs.append((y, mean, rstd, saved.values, saved.exponents, dx, dw, db))
        assert all(torch.equal(p, q) for p, q in zip(*runs))


def test_streams_and_graphs():
    import paper_2402_11857_amd as pkg

    say("case group norm on another stream and captured")
    shape, G = (3, 2, 300, 80), 5
    x, dy, w, b = _inputs(shape, "bf16", seed=16)

    def both():
        y, mean, rstd, saved = pkg.liec_group_norm(x, G, w, b, activation="silu", save=True)
        dw, db = torch.empty_like(w), torch.empty_like(b)
        dx = pkg.liec_group_norm_backward(dy, saved, mean, rstd, w, b, activation="silu", dweight=dw, dbias=db)
        return y, mean, rstd, dx, dw, db

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    # two graphs of the same pool, replayed in turn with eager calls between them
    graphs, outputs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            outputs.append(both())
        graphs.append(graph)
    for i in range(4):
        x.copy_(activations(shape, "bf16", seed=30 + i))
        want = both()
        for graph, out in zip(graphs, outputs):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(want, out)), i
            both()


def test_large_offsets():
    import paper_2402_11857_amd as pkg

    say("case group norm of 2^31 + 2^25 values")
    N, B, S, C, G = 2, 1, 32_800, 32_768, 8
    x = torch.empty(N, B, S, C, dtype=torch.bfloat16, device=DEV).normal_(0.5, 1.0, generator=generator(17))
    y, mean, rstd = pkg.liec_group_norm(x, G, out=x.clone())
    for g in (0, G - 1):
        v = x[1, 0, :, g * 4096:(g + 1) * 4096].float()
        mu, sd = v.double().mean(), v.double().std(correction=0)
        assert abs(float(mean[1, 0, g]) - float(mu)) < 1e-5 and abs(float(rstd[1, 0, g]) * float(sd) - 1) < 1e-5
        want = ((v[-1].double() - mu) / sd)
        assert float((y[1, 0, -1, g * 4096:(g + 1) * 4096].double() - want).abs().max()) < 2 ** -8 * 6


@pytest.mark.parametrize("N,B", [(3, 3001), (1, 9001), (2, 8500)])
def test_many_images_in_parts(N, B):
    """More partial sums than the scratch holds at a time: whole workers, or some of one worker's images; images that blocks hold,
    and others."""
    import paper_2402_11857_amd as pkg

    say(f"case group norm of {N} x {B} images")
    for S, C, G in ((2, 4096, 32), (2, 4100, 1)):            # 4100 channels in one group: no block holds it
        x, dy, w, b = _inputs((N, B, S, C), "bf16", seed=21)
        y, mean, rstd, saved = pkg.liec_group_norm(x, G, w, b, activation="silu", save=True)
        check_forward(x, G, w, b, "silu", y, mean, rstd)
        for shape, at in (((N, C), x), ((C,), saved)):
            dw, db = torch.full(shape, 9.0, device=DEV), torch.full(shape, 9.0, device=DEV)
            dx = pkg.liec_group_norm_backward(dy, at, mean, rstd, w, b, activation="silu", dweight=dw, dbias=db)
            check_backward(dy, at if at is x else value(saved), mean, rstd, G, w, b, "silu", dx, dw, db)
            assert torch.equal(dx[0, -1], pkg.liec_group_norm_backward(dy[:1, -1:], at[:1, -1:] if at is x else pkg.Checkpoint(*(t[:1, -1:].contiguous() for t in at)),
                                                                       mean[:1, -1:].contiguous(), rstd[:1, -1:].contiguous(), w[:1], b[:1], activation="silu")[0, 0])


def test_refusals():
    import paper_2402_11857_amd as pkg

    say("case group norm refusals")
    x, dy, w, b = _inputs((2, 3, 5, 24), "fp32", seed=18)
    y, mean, rstd, saved = pkg.liec_group_norm(x, 3, w, b, save=True)
    for error, call in ((ValueError, lambda: pkg.liec_group_norm(x[0, 0], 3)), (ValueError, lambda: pkg.liec_group_norm(x, 5)), (ValueError, lambda: pkg.liec_group_norm(x, 0)),
                        (TypeError, lambda: pkg.liec_group_norm(x, 1.5)), (TypeError, lambda: pkg.liec_group_norm(x.double(), 3)),
                        (ValueError, lambda: pkg.liec_group_norm(x, 3, w[:1])), (ValueError, lambda: pkg.liec_group_norm(x, 3, w[:, :23])),
                        (TypeError, lambda: pkg.liec_group_norm(x, 3, w, b.half())), (TypeError, lambda: pkg.liec_group_norm(x, 3, w.cpu())),
                        (ValueError, lambda: pkg.liec_group_norm(x.transpose(2, 3), 5)), (ValueError, lambda: pkg.liec_group_norm(x, 3, out=y[:1])),
                        (TypeError, lambda: pkg.liec_group_norm(x, 3, out=y.half())), (pkg.LiecError, lambda: pkg.liec_group_norm(x, 3, eps=-1.0)),
                        (pkg.LiecError, lambda: pkg.liec_group_norm(x, 3, out=x.flip(0).flip(0)[:, :, :1].expand_as(x))),
                        (TypeError, lambda: pkg.liec_group_norm_backward(dy, None, mean, rstd)), (TypeError, lambda: pkg.liec_group_norm_backward(dy, x.half(), mean, rstd)),
                        (ValueError, lambda: pkg.liec_group_norm_backward(dy, x[:, :2], mean, rstd)), (TypeError, lambda: pkg.liec_group_norm_backward(dy, x, mean[:, :2], rstd)),
                        (TypeError, lambda: pkg.liec_group_norm_backward(dy, x, mean, rstd[..., :1])), (TypeError, lambda: pkg.liec_group_norm_backward(dy, x, mean.half(), rstd)),
                        (ValueError, lambda: pkg.liec_group_norm_backward(dy[:, :, :4], saved, mean, rstd)),
                        (ValueError, lambda: pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, dweight=torch.zeros(1, 24, device=DEV).expand(2, 24))),
                        (pkg.LiecError, lambda: pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, dweight=w)),
                        (pkg.LiecError, lambda: pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, dweight=y[0, 0, :2], dbias=torch.empty(24, device=DEV))),
                        (ValueError, lambda: pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, dweight=torch.empty(2, 23, device=DEV)))):
        with pytest.raises(error):
            call()


def test_written_tensors_change_their_version():
    import paper_2402_11857_amd as pkg

    say("case group norm versions")
    x, dy, w, b = _inputs((2, 3, 5, 24), "fp32", seed=19)
    out, dx, dw, db = (torch.empty_like(t) for t in (x, x, w, b))
    before = [t._version for t in (out, dx, dw, db, x, dy, w)]
    _, mean, rstd = pkg.liec_group_norm(x, 3, w, b, out=out)
    pkg.liec_group_norm_backward(dy, x, mean, rstd, w, b, dx=dx, dweight=dw, dbias=db)
    assert [t._version > v for t, v in zip((out, dx, dw, db, x, dy, w), before)] == [True] * 4 + [False] * 3
    assert not pkg.liec_group_norm(x.requires_grad_(), 3)[0].requires_grad
