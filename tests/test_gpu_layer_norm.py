"""Layer normalisation and its gradients against the definitions in 64 bits.

Bounds, with u = 2^-24 and chains of at most 64 fp32 additions per sum of a row (16 values of a lane, 6 steps inside a wave,
16 waves): the mean is off by at most 64 u max|x|, the variance by 64 u relative and that squared; normalised values, products
and shifts add a few u; the result is rounded once to its type.  Weight gradients add up over rows, in chains of at most
min(rows, 256) + 64 additions."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402
from _train import DTYPES, TINY, U, U32, assert_within, generator  # noqa: E402

pytestmark = GPU_MARKS
EPS = 1e-5


def _name(dtype):
    return next(k for k, v in DTYPES.items() if v == dtype)


def _inputs(shape, dtype, seed, params="fp32", offset=0.3):
    gen = generator(seed)
    N, C = shape[0], shape[-1]
    x = (torch.randn(shape, generator=gen, device=DEV) * (0.25 + 2 * torch.rand(C, generator=gen, device=DEV)) + offset).to(DTYPES[dtype])
    dy = (torch.randn(shape, generator=gen, device=DEV) * 0.1).to(DTYPES[dtype])
    w = (1 + 0.1 * torch.randn(N, C, generator=gen, device=DEV)).to(DTYPES[params])
    b = (0.1 * torch.randn(N, C, generator=gen, device=DEV)).to(DTYPES[params])
    return x, dy, w, b


def _spread(p, x):
    """[C] or [N, C] parameters in 64 bits, shaped to go with x."""
    p = p.double()
    return p.reshape(p.shape[0], *([1] * (x.dim() - 2)), p.shape[1]) if p.dim() == 2 else p


def _check_forward(x, w, b, eps, y, mean, rstd):
    v = x.double()
    mu = v.mean(-1, keepdim=True)
    var = (v - mu).square().mean(-1, keepdim=True)
    rs = 1 / torch.sqrt(var + eps)
    h = (v - mu) * rs
    A = v.abs().amax(-1, keepdim=True)
    off_mu = 64 * U32 * A
    off_var = 70 * U32 * var + off_mu ** 2 + 2 * U32 * eps
    off_rs = rs * (0.5 * off_var / (var + eps) * 1.01 + 3 * U32)
    assert mean.dtype == rstd.dtype == torch.float32
    assert_within(mean, mu[..., 0], off_mu[..., 0] + 1e-45, "mean")
    assert_within(rstd, rs[..., 0], off_rs[..., 0], "rstd")
    wd = _spread(w, x) if w is not None else torch.ones((), dtype=torch.float64, device=x.device)
    bd = _spread(b, x) if b is not None else torch.zeros((), dtype=torch.float64, device=x.device)
    want = h * wd + bd
    t = _name(x.dtype)
    bound = wd.abs() * (off_mu * rs + h.abs() * (off_rs / rs + 3 * U32)) * 1.01 + 2 * U32 * want.abs()
    if t != "fp32":
        bound = bound + 1.01 * U[t] * (want.abs() + bound)
    assert_within(y, want, bound + TINY[t], "y")


def _check_backward(dy, x, mean, rstd, w, dx, dw, db):
    g, mu, rs = dy.double(), mean.double()[..., None], rstd.double()[..., None]
    h = (x.double() - mu) * rs
    wd = _spread(w, x) if w is not None else torch.ones((), dtype=torch.float64, device=x.device)
    a = g * wd
    m1, m2 = a.mean(-1, keepdim=True), (a * h).mean(-1, keepdim=True)
    t = _name(x.dtype)
    if dx is not None:
        want = rs * (a - m1 - h * m2)
        A1, A2 = a.abs().mean(-1, keepdim=True), (a * h).abs().mean(-1, keepdim=True)
        bound = rs * (6 * U32 * (a.abs() + m1.abs() + (h * m2).abs()) + 70 * U32 * (A1 + h.abs() * A2))
        if t != "fp32":
            bound = bound + 1.01 * U[t] * (want.abs() + bound)
        assert_within(dx, want, bound + TINY[t], "dx")
    for got, term, what in ((dw, g * h, "dweight"), (db, g, "dbias")):
        if got is None:
            continue
        if got.dim() == 2:
            term = term.reshape(got.shape[0], -1, term.shape[-1])
            want, mass, rows = term.sum(1), term.abs().sum(1), term.shape[1]
        else:
            term = term.reshape(-1, term.shape[-1])
            want, mass, rows = term.sum(0), term.abs().sum(0), term.shape[0]
        p = _name(got.dtype)
        bound = (min(rows, 256) + 64) * U32 * mass
        if p != "fp32":
            bound = bound + 1.01 * U[p] * (want.abs() + bound)
        assert_within(got, want, bound + TINY[p], what)


def _both(x, dy, w, b, eps=EPS):
    import paper_2402_11857_amd as pkg

    y, mean, rstd = pkg.liec_layer_norm(x, w, b, eps)
    _check_forward(x, w, b, eps, y, mean, rstd)
    dw, db = (None if w is None else torch.full_like(w, 9.0)), (None if b is None else torch.full_like(b, 9.0))
    dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)
    _check_backward(dy, x, mean, rstd, w, dx, dw, db)


# both sides of every change of the team that holds a row, odd lengths, rows too short and too long to be held
COLUMNS = [1, 2, 7, 8, 9, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 1001, 1024, 1025, 2048, 2049, 4095, 4096, 4097,
           8191, 8192, 8193, 16383, 16384, 16385, 40_003]


@pytest.mark.parametrize("C", COLUMNS)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_every_row_length(C, dtype):
    say(f"case layer norm C={C} {dtype}")
    for N, R in ((1, 1), (3, 5), (2, 67)):
        _both(*_inputs((N, R, C), dtype, seed=C + R))


@pytest.mark.parametrize("N,R,C", [(1, 5000, 64), (1, 3000, 24), (7, 1030, 40), (2, 4097, 257), (1, 9001, 1001), (5, 300, 4096), (70, 33, 130),
                                   (1, 2000, 8200), (3, 513, 16_384), (1, 3001, 4100), (1, 2500, 4096), (1, 6001, 2048), (1, 1501, 8192),
                                   (1, 5003, 1024), (2, 20_001, 16), (1, 12_007, 512), (2, 700, 20_000), (3, 700, 5), (1, 70_001, 5)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_many_rows(N, R, C, dtype):
    say(f"case layer norm N={N} R={R} C={C} {dtype}")
    _both(*_inputs((N, R, C), dtype, seed=R))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("params", list(DTYPES))
def test_types_of_weights(dtype, params):
    say(f"case layer norm {dtype} with weights in {params}")
    for C in (5, 96, 1027, 17_000):
        _both(*_inputs((3, 9, C), dtype, seed=C, params=params))


def test_weights_shared_by_all_workers_or_missing():
    import paper_2402_11857_amd as pkg

    say("case layer norm, shared and missing weights")
    for C in (5, 100, 1500, 17_000):
        x, dy, w, b = _inputs((4, 37, C), "bf16", seed=21)
        _both(x, dy, w[0], b[0])
        _both(x, dy, None, None)
        _both(x, dy, w, None)
        _both(x, dy, None, b)
        _both(x[0], dy[0], w[0], b[0])                       # [rows, C]
        _both(x.view(2, 2, 37, C), dy.view(2, 2, 37, C), w[0], b[0])
        _both(x[:, 0].contiguous(), dy[:, 0].contiguous(), w, b)       # one row per worker
        # a weight that all workers share, with a gradient of each worker's own
        y, mean, rstd = pkg.liec_layer_norm(x, w[0])
        dw = torch.empty(4, C, device=DEV)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w[0], dweight=dw)
        _check_backward(dy, x, mean, rstd, w[0], dx, dw, None)
        db = torch.empty(4, C, device=DEV)
        assert pkg.liec_layer_norm_backward(dy, x, mean, rstd, w[0], dbias=db, need_dx=False) is None
        _check_backward(dy, x, mean, rstd, w[0], None, None, db)


def test_strides():
    import paper_2402_11857_amd as pkg

    say("case layer norm, strides")
    for C in (6, 40, 1001, 17_001):
        base, dbase, w, b = _inputs((3, 11, C + 7), "fp16", seed=31)
        rows = torch.randn(3, 2 * C + 19, generator=generator(32), device=DEV)
        wv, bv = rows[:, 3:3 + C], rows[:, 5 + C:5 + 2 * C]                          # columns of a models tensor
        grads = torch.full((3, 2 * C + 19), 5.0, device=DEV)
        gw, gb = grads[:, 3:3 + C], grads[:, 5 + C:5 + 2 * C]
        x, dy = base[:, :, 3:3 + C], dbase[:, :, 1:1 + C]                            # rows at distances of C + 7
        y, mean, rstd = pkg.liec_layer_norm(x, wv, bv, EPS)
        _check_forward(x, wv, bv, EPS, y, mean, rstd)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, wv, dweight=gw, dbias=gb)
        _check_backward(dy, x, mean, rstd, wv, dx, gw, gb)
        rest = torch.ones(2 * C + 19, dtype=torch.bool, device=DEV)
        rest[3:3 + C] = rest[5 + C:5 + 2 * C] = False
        assert bool((grads[:, rest] == 5.0).all())
        # rows outermost: [R, N, C] seen as [N, R, C]; output and gradient laid out alike
        xt, dyt = base.transpose(0, 1).contiguous().transpose(0, 1)[..., :C], dbase.transpose(0, 1).contiguous().transpose(0, 1)[..., :C]
        out = torch.full_like(base, 3.0).transpose(0, 1).contiguous().transpose(0, 1)
        y, mean, rstd = pkg.liec_layer_norm(xt, wv, bv, EPS, out=out[..., :C])
        _check_forward(xt, wv, bv, EPS, y, mean, rstd)
        assert bool((out[..., C:] == 3.0).all())
        dx = pkg.liec_layer_norm_backward(dyt, xt, mean, rstd, wv, dx=out[..., :C], dweight=gw, dbias=gb)
        _check_backward(dyt, xt, mean, rstd, wv, dx, gw, gb)
        assert bool((out[..., C:] == 3.0).all())
        # one weight, activations contiguous, their gradient not
        xc = x.contiguous()
        y, mean, rstd = pkg.liec_layer_norm(xc, wv[0], bv[0], EPS)
        dw = torch.empty(C, device=DEV)
        dx = pkg.liec_layer_norm_backward(dy, xc, mean, rstd, wv[0], dweight=dw)
        _check_backward(dy, xc, mean, rstd, wv[0], dx, dw, None)


@pytest.mark.parametrize("C", [5, 129, 1001, 4100, 17_001])
def test_in_place(C):
    import paper_2402_11857_amd as pkg

    say(f"case layer norm in place C={C}")
    x, dy, w, b = _inputs((2, 300, C), "bf16", seed=41)
    y, mean, rstd = pkg.liec_layer_norm(x, w, b)
    again = x.clone()
    out, mean2, rstd2 = pkg.liec_layer_norm(again, w, b, out=again)
    assert out is again and torch.equal(again, y) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    dw, db, dw2, db2 = (torch.empty_like(w) for _ in range(4))
    dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)
    for take in (0, 1):
        gy, gx = dy.clone(), x.clone()
        got = pkg.liec_layer_norm_backward(gy, gx, mean, rstd, w, dx=(gy, gx)[take], dweight=dw2, dbias=db2)
        assert torch.equal(got, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_gradients_against_differences():
    import paper_2402_11857_amd as pkg

    say("case layer norm, gradients against differences")
    for C in (6, 50, 700, 17_003):
        x, dy, w, b = _inputs((2, 4, C), "fp32", seed=51)
        _, mean, rstd = pkg.liec_layer_norm(x, w, b)
        dw, db = torch.empty_like(w), torch.empty_like(b)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)

        def loss(xv, wv, bv):
            mu = xv.mean(-1, keepdim=True)
            var = (xv - mu).square().mean(-1, keepdim=True)
            return (((xv - mu) / torch.sqrt(var + EPS) * wv[:, None] + bv[:, None]) * dy.double()).sum()

        gen = generator(52)
        for i, grad in enumerate((dx, dw, db)):
            point = [x.double(), w.double(), b.double()]
            step = torch.randn(grad.shape, generator=gen, device=DEV, dtype=torch.float64) * 1e-4
            hi, lo = list(point), list(point)
            hi[i], lo[i] = point[i] + step, point[i] - step
            slope = (loss(*hi) - loss(*lo)) / 2
            got = (grad.double() * step).sum()
            # the third-order term of the difference, and the gradients' own rounding
            scale = float((grad.double() * step).abs().sum())
            assert abs(float(slope - got)) <= 1e-5 * scale + 1e-9, (C, i, float(slope), float(got), scale)


def test_rows_that_are_constant_or_not_finite():
    import paper_2402_11857_amd as pkg

    say("case layer norm, constant rows, Inf and NaN")
    for C in (6, 100, 3000, 17_000):
        x, dy, w, b = _inputs((2, 6, C), "fp32", seed=61)
        x[0, 1] = 4.0
        x[0, 2] = 0.0
        x[1, 3, C // 2] = float("nan")
        x[1, 4, C - 1] = float("inf")
        y, mean, rstd = pkg.liec_layer_norm(x, w, b)
        assert_within(y[0, 1:3], b[0].double().expand(2, C), torch.tensor(1e-3 if C > 16_384 else 64 * U32 * 4 * 400, device=DEV), "constant rows")
        assert y[1, 3:5].isnan().any(-1).all() and rstd[1, 3].isnan() and not rstd[1, 4].isfinite()
        good = torch.tensor([0, 1, 2, 5], device=DEV)
        _check_forward(x[1, good], w[1], b[1], EPS, y[1, good], mean[1, good], rstd[1, good])
        dw, db = torch.empty_like(w), torch.empty_like(b)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)
        _check_backward(dy[:1], x[:1], mean[:1], rstd[:1], w[:1], dx[:1], dw[:1], db[:1])     # the other worker's trouble is its own
        assert dw[1].isnan().any() and db[1].isfinite().all() and dx[1, 3].isnan().all()
        # no variance at all and no eps: what 1 / sqrt(0) gives
        y, mean, rstd = pkg.liec_layer_norm(torch.zeros(1, C, device=DEV), eps=0.0)
        assert rstd.isinf().all() and y.isnan().all()


def test_a_mean_far_larger_than_the_spread():
    import paper_2402_11857_amd as pkg

    say("case layer norm, large mean")
    for C in (100, 1000, 5000, 17_000):
        x, _, w, b = _inputs((1, 20, C), "fp32", seed=71, offset=1000.0)
        _check_forward(x, w, b, EPS, *pkg.liec_layer_norm(x, w, b))


def test_no_rows():
    import paper_2402_11857_amd as pkg

    say("case layer norm, no rows")
    for C in (4, 100, 17_000):
        x, w = torch.empty(3, 0, C, device=DEV), torch.ones(3, C, device=DEV)
        y, mean, rstd = pkg.liec_layer_norm(x, w, w)
        assert y.shape == x.shape and mean.shape == rstd.shape == (3, 0)
        for shape in ((3, C), (C,)):
            dw, db = torch.full(shape, 9.0, device=DEV), torch.full(shape, 9.0, device=DEV)
            dx = pkg.liec_layer_norm_backward(x, x, mean, rstd, w[0], dweight=dw, dbias=db)
            assert dx.shape == x.shape and bool((dw == 0).all()) and bool((db == 0).all())


def test_activations_beyond_32_bit_offsets():
    import paper_2402_11857_amd as pkg

    R, C = (1 << 20) + 3, 2056
    say(f"case layer norm, {R} rows of {C} columns")
    x = torch.zeros(R, C, dtype=torch.bfloat16, device=DEV)
    last = _inputs((1, 40, C), "bf16", seed=81)
    x[-40:] = last[0][0]
    y, mean, rstd = pkg.liec_layer_norm(x)
    _check_forward(x[-40:], None, None, EPS, y[-40:], mean[-40:], rstd[-40:])
    assert bool((y[:-40:4096] == 0).all())
    dy = torch.zeros_like(x)
    dy[-40:] = last[1][0]
    dw = torch.empty(C, device=DEV)
    pkg.liec_layer_norm_backward(dy, x, mean, rstd, dx=y, dweight=dw)
    _check_backward(dy[-40:], x[-40:], mean[-40:], rstd[-40:], None, y[-40:], dw, None)


def test_another_stream_and_graph_replays():
    import paper_2402_11857_amd as pkg

    say("case layer norm on another stream, in a graph")
    x, dy, w, b = _inputs((3, 50, 700), "bf16", seed=91)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, mean, rstd = pkg.liec_layer_norm(x, w, b)
        dw, db = torch.empty_like(w), torch.empty_like(b)
        dx = pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)
    side.synchronize()
    _check_forward(x, w, b, EPS, y, mean, rstd)
    _check_backward(dy, x, mean, rstd, w, dx, dw, db)
    want = [t.clone() for t in (dx, dw, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dx=dx, dweight=dw, dbias=db)
    for k in range(3):
        for t in (dx, dw, db):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((dx, dw, db), want)), f"replay {k}"


def test_c_entry_points_without_statistics_and_with_rows_in_reverse():
    import ctypes

    import paper_2402_11857_amd as pkg
    from test_train_abi import Param, Rows

    say("case layer norm through the C entry points")
    lib, ref, N, R = pkg.lib(), ctypes.byref, 2, 7
    for C in (5, 200, 5000, 17_000):
        x, _, w, b = _inputs((N, R, C), "fp32", seed=111)
        y = torch.full((N, R, C), 9.0, device=DEV)
        # rows from the last to the first, of the last worker first
        xr = Rows(x.data_ptr() + 4 * (N * R - 1) * C, -R * C, -C)
        yr = Rows(y.data_ptr() + 4 * (N * R - 1) * C, -R * C, -C)
        wr, br = Param(w.data_ptr() + 4 * C, -C), Param(b.data_ptr() + 4 * C, -C)
        stream = torch.cuda.current_stream().cuda_stream
        assert lib.liec_layer_norm(ref(xr), ref(wr), ref(br), ref(yr), None, None, N, R, C, EPS, 0, 0, stream) == 0
        want, mean, rstd = pkg.liec_layer_norm(x, w, b, EPS)
        assert torch.equal(y, want)
        dw = torch.full((N, C), 9.0, device=DEV)
        dr = Param(dw.data_ptr() + 4 * C, -C)
        need = lib.liec_layer_norm_workspace(N, R, C)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
        m, r = mean.flip(0, 1).contiguous(), rstd.flip(0, 1).contiguous()
        assert lib.liec_layer_norm_backward(ref(xr), ref(xr), m.data_ptr(), r.data_ptr(), ref(wr), None, ref(dr), None, N, R, C, 0, 0,
                                            ws.data_ptr(), need, stream) == 0
        _check_backward(x, x, mean, rstd, w, None, dw, None)


def test_refusals():
    import paper_2402_11857_amd as pkg

    say("case layer norm, refusals")
    x, dy, w, b = _inputs((2, 4, 64), "fp32", seed=101)
    y, mean, rstd = pkg.liec_layer_norm(x, w, b)
    for bad in (lambda: pkg.liec_layer_norm(x.cpu()),
                lambda: pkg.liec_layer_norm(x.double()),
                lambda: pkg.liec_layer_norm(x, w.double()),
                lambda: pkg.liec_layer_norm(x, w, b.bfloat16()),
                lambda: pkg.liec_layer_norm(x, w, out=y.half()),
                lambda: pkg.liec_layer_norm_backward(dy.half(), x, mean, rstd, w),
                lambda: pkg.liec_layer_norm_backward(dy, x, mean.double(), rstd, w),
                lambda: pkg.liec_layer_norm_backward(dy, x, mean[:1], rstd, w)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: pkg.liec_layer_norm(x, w[:, :63]),
                lambda: pkg.liec_layer_norm(x, torch.ones(3, 64, device=DEV)),
                lambda: pkg.liec_layer_norm(x[..., ::2], w[:, ::2].contiguous()),
                lambda: pkg.liec_layer_norm(x, w, out=y[:1]),
                lambda: pkg.liec_layer_norm(torch.empty(4, 0, device=DEV)),
                lambda: pkg.liec_layer_norm(x, torch.empty(0, 64, device=DEV)),
                lambda: pkg.liec_layer_norm_backward(dy[:1], x, mean, rstd, w)):
        with pytest.raises(ValueError):
            bad()
    flat = torch.zeros(2 * 4 * 64 + 8, device=DEV)
    for bad in (lambda: pkg.liec_layer_norm(x, w, b, eps=-1.0),
                lambda: pkg.liec_layer_norm(x, w, b, eps=float("inf")),
                lambda: pkg.liec_layer_norm(flat[:512].view(2, 4, 64), w, out=flat[8:].view(2, 4, 64)),          # they overlap
                lambda: pkg.liec_layer_norm(x, w, out=torch.empty(2, 1, 64, device=DEV).expand(2, 4, 64)),
                lambda: pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dx=torch.empty(1, 4, 64, device=DEV).expand(2, 4, 64)),
                lambda: pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=w, dbias=w),
                lambda: pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=torch.empty(2, 64, device=DEV), dbias=torch.empty(64, device=DEV))):
        with pytest.raises(pkg.LiecError):
            bad()
