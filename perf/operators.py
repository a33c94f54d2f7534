"""What the speed of the operators around a backward pass is measured on: the layers' normalisation and its gradients, the
global norm of a worker's gradient tensors, and clipping, in place or on the way into the rows that a compressed step reads.

`run` computes a case in elementary torch operations, or, with `own` set, through the framework's entry points.  Every
worker has a model of its own, so weights are rows of a models tensor and each worker's weight gradient is a reduction over
that worker's rows only.  Inputs are seeded: gradients of per-tensor scales with heavy-tailed outliers, activations with an
offset and channels of unequal size.
"""
from __future__ import annotations

import math

import torch

own = False

R18, R50, VGG = 11_689_512, 25_557_032, 138_357_544     # elements of a worker's model: ResNet-18, ResNet-50, VGG-16
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5
FALL = 0.9999        # an in-place clip's bound falls by this from pass to pass, so that every pass has something to clip


# ---- sizes -----------------------------------------------------------------------------------------------------------
def _norm_pair(c):
    return [c, c]


def _r18():
    """Parameter tensors of ResNet-18: 20 convolutions, a scale and a shift after each, one linear layer."""
    stage = lambda i, c: [x for b in range(2) for x in (                                            # noqa: E731
        [(i if b == 0 else c) * c * 9] + _norm_pair(c) + [c * c * 9] + _norm_pair(c) +
        ([i * c] + _norm_pair(c) if b == 0 and i != c else []))]
    return [9408] + _norm_pair(64) + stage(64, 64) + stage(64, 128) + stage(128, 256) + stage(256, 512) + [512_000, 1000]


def _r50():
    """Parameter tensors of ResNet-50: 53 convolutions, a scale and a shift after each, one linear layer."""
    block = lambda i, c, b: ([(i if b == 0 else 4 * c) * c] + _norm_pair(c) + [9 * c * c] + _norm_pair(c) + [4 * c * c] +   # noqa: E731
                             _norm_pair(4 * c) + ([i * 4 * c] + _norm_pair(4 * c) if b == 0 else []))
    return [9408] + _norm_pair(64) + [x for i, c, n in ((64, 64, 3), (256, 128, 4), (512, 256, 6), (1024, 512, 3))
                                      for b in range(n) for x in block(i, c, b)] + [2_048_000, 1000]


def _vgg():
    """Parameter tensors of VGG-16: 13 convolutions and 3 linear layers, each with a bias."""
    c = (3, 64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512)
    return [x for i, o in zip(c, c[1:]) for x in (9 * i * o, o)] + [102_760_448, 4096, 16_777_216, 4096, 4_096_000, 1000]


NETS = {"r18": _r18, "r50": _r50, "vgg": _vgg, "equal": lambda: [1] * 16}


def _sizes(case):
    """The tensors' lengths: those of the named architecture, scaled to d elements in all."""
    full, d = NETS[case["net"]](), case["d"]
    sizes = [max(1, s * d // sum(full)) for s in full]
    at = sizes.index(max(sizes))
    sizes[at] += d - sum(sizes)
    return sizes


# ---- cases -----------------------------------------------------------------------------------------------------------
def _grads(what, N, d, net, dtype, **kw):
    return dict(kw, what=what, N=N, d=d, net=net, dtype=dtype)


def _layer(what, N, R, C, dtype, **kw):
    return dict(kw, what=what, N=N, R=R, C=C, dtype=dtype)


def listed():
    return [
        # the norm that a run logs at every step of the smallest simulation: launches and latency
        _grads("norm", 4, 65_536, "equal", "fp32", name="norm_tiny"),
        # the same of 32 workers, 161 tensors each, out of a bf16 backward pass
        _grads("norm", 32, R50, "r50", "bf16", name="norm_r50_bf16"),
        # clipping in place: a model of odd length in fp16 (loss-scaled), 32 tensors, an odd number of workers
        _grads("clip", 5, 3_000_017, "vgg", "fp16", name="clip_ragged_fp16"),
        # clipping in place of 16 workers' fp32 gradients, 62 tensors
        _grads("clip", 16, R18, "r18", "fp32", name="clip_r18"),
        # bf16 gradients clipped into the fp32 rows of the mid-sized top-k run, everything in caches
        _grads("gather", 8, 1_048_576, "equal", "bf16", name="gather_mid"),
        # the largest: 16 workers' bf16 gradients, most of each in one tensor, clipped into their rows
        _grads("gather", 16, VGG, "vgg", "bf16", name="gather_vgg"),
        # one token per worker through a normalisation: latency
        _layer("forward", 4, 1, 1024, "bf16", name="ln_token"),
        # rows of odd length, off any alignment, fp16
        _layer("forward", 5, 333, 1001, "fp16", name="ln_ragged_fp16"),
        # a training batch: 8 workers of 8192 tokens
        _layer("forward", 8, 8192, 4096, "bf16", name="ln_large"),
        # gradients of a small fp32 layer
        _layer("backward", 4, 32, 256, "fp32", name="ln_grad_tiny"),
        # many workers with few rows each: weight gradients are a large share of the work
        _layer("backward", 16, 512, 1024, "bf16", name="ln_grad_mid"),
        # a training batch: 8 workers of 8192 tokens
        _layer("backward", 8, 8192, 4096, "bf16", name="ln_grad_large"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """Gradients: 1 to 64 workers of 2^14 to 1.4e8 elements, at most 4e8 in all; layers: 1 to 32 workers, rows of 16 to 16384
    columns, at most 2.6e8 elements in all; any remainder, each type."""
    what = rng.choice(("norm", "clip", "gather", "forward", "backward"))
    dtype = rng.choice(("fp32", "bf16", "fp16"))
    if what in ("forward", "backward"):
        N, C = _log_uniform(rng, 1, 32), _log_uniform(rng, 16, 16_384)
        C += C == 3072
        return _layer(what, N, _log_uniform(rng, 1, 260_000_000 // (N * C)), C, dtype)
    N = _log_uniform(rng, 1, 64)
    return _grads(what, N, _log_uniform(rng, 16_384, min(VGG, 400_000_000 // N)), rng.choice(tuple(NETS)), dtype)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _gradients(case, seed):
    """One buffer with all tensors one after the other, the tensors as its views [N, n_t], and the bound of the norms."""
    N, sizes, dtype = case["N"], _sizes(case), TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    scale = 10.0 ** (2.0 * torch.rand(len(sizes), generator=gen, device="cuda") - (1.0 if case["dtype"] == "fp16" else 3.0))
    worker = 0.5 + 1.5 * torch.rand(N, 1, generator=gen, device="cuda")
    buffer = torch.empty(N * case["d"], dtype=dtype, device="cuda")
    tensors, squares, at = [], torch.zeros(N, device="cuda"), 0
    for t, n in enumerate(sizes):
        g = buffer[at:at + N * n].view(N, n)
        at += N * n
        g.normal_(generator=gen)
        few = torch.randint(0, n, (max(1, n // 1000),), generator=gen, device="cuda")      # one in a thousand is an outlier
        g[:, few] *= 8.0
        g.mul_(scale[t] * worker)
        squares += (g.float() ** 2).sum(1)
        tensors.append(g)
    norms = squares.sqrt()
    # in place every worker is clipped, into the rows about half of them are
    bound = 0.25 * norms.min() if case["what"] == "clip" else norms.median()
    return buffer, tensors, float(bound)


def _activations(case, seed):
    """x and the gradient of y, [N, R, C]; weights and biases as columns of a models tensor; gradient rows of its shape."""
    N, R, C, dtype = case["N"], case["R"], case["C"], TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    channel = 0.25 + 2.0 * torch.rand(C, generator=gen, device="cuda")
    x = torch.empty((N, R, C), dtype=dtype, device="cuda").normal_(0.3, 1.0, generator=gen).mul_(channel)
    dy = torch.empty((N, R, C), dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=gen) if case["what"] == "backward" else None
    models = torch.empty((N, 2 * C + 101), device="cuda").normal_(0.0, 0.1, generator=gen)
    models[:, 37:37 + C] += 1.0
    return x, dy, models


def _columns(rows, C):
    """The weight's and the bias's columns of a worker's row."""
    return rows[:, 37:37 + C], rows[:, 37 + C:37 + 2 * C]


def prepare(case, seed):
    if case["what"] in ("norm", "clip", "gather"):
        buffer, tensors, bound = _gradients(case, seed)
        rows = torch.empty((case["N"], case["d"]), device="cuda") if case["what"] == "gather" else None
        return dict(case=case, buffer=buffer, tensors=tensors, bound=bound, rows=rows,
                    norms=torch.empty(case["N"], device="cuda"))
    x, dy, models = _activations(case, seed)
    state = dict(case=case, x=x, dy=dy)
    state["weight"], state["bias"] = _columns(models, case["C"])
    if dy is not None:                                       # what the forward pass kept, and the rows that take the gradients
        wide = x.float()
        mean = wide.mean(2)
        state["rstd"] = ((wide - mean[..., None]).square().mean(2) + EPS).rsqrt()
        state["mean"] = mean
        state["dweight"], state["dbias"] = _columns(torch.zeros_like(models), case["C"])
    return state


# ---- one pass --------------------------------------------------------------------------------------------------------
def _framework(state):
    import paper_2402_11857_amd as liec

    what = state["case"]["what"]
    if what == "norm":
        return liec.liec_grad_norm(state["tensors"], state["norms"])
    if what == "clip":
        liec.liec_clip_grads(state["tensors"], state["bound"], state["norms"])
        state["bound"] *= FALL
        return state["buffer"], state["norms"]
    if what == "gather":
        liec.liec_gather_grads(state["tensors"], state["rows"], state["bound"], state["norms"])
        return state["rows"], state["norms"]
    if what == "forward":
        return liec.liec_layer_norm(state["x"], state["weight"], state["bias"], EPS)
    dx = liec.liec_layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["weight"],
                                       dweight=state["dweight"], dbias=state["dbias"])
    return dx, state["dweight"], state["dbias"]


def run(state):
    if own:
        return _framework(state)
    what = state["case"]["what"]
    if what in ("norm", "clip", "gather"):
        tensors = state["tensors"]
        norms = torch.stack([t.float().square().sum(1) for t in tensors]).sum(0).sqrt()
        if what == "norm":
            return norms
        factor = torch.where(norms <= state["bound"], torch.ones_like(norms), state["bound"] / norms)[:, None]
        if what == "gather":
            columns = torch.split(state["rows"], [t.shape[1] for t in tensors], 1)
            [c.copy_(t.float() * factor) for c, t in zip(columns, tensors)]
            return state["rows"], norms
        [t.copy_(t.float() * factor) for t in tensors]
        state["bound"] *= FALL
        return state["buffer"], norms
    x, w = state["x"].float(), state["weight"][:, None, :]
    if what == "forward":
        mean = x.mean(2)
        x = x - mean[..., None]
        rstd = 1.0 / torch.sqrt((x * x).mean(2) + EPS)
        y = x * rstd[..., None] * w + state["bias"][:, None, :]
        return y.to(state["x"].dtype), mean, rstd
    dy, rstd = state["dy"].float(), state["rstd"][..., None]
    xhat = (x - state["mean"][..., None]) * rstd
    state["dbias"].copy_(dy.sum(1))
    state["dweight"].copy_((dy * xhat).sum(1))
    dy = dy * w
    dx = rstd * (dy - dy.mean(2, keepdim=True) - xhat * (dy * xhat).mean(2, keepdim=True))
    return dx.to(state["x"].dtype), state["dweight"], state["dbias"]


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["what"] in ("norm", "clip", "gather"):
        n = case["N"] * case["d"]
        written = {"norm": 0, "clip": size * n, "gather": 4 * n}[case["what"]]
        return {"bytes": size * n + written + 4 * case["N"], "flops": (2 if case["what"] == "norm" else 3) * n}
    rows, n = case["N"] * case["R"], case["N"] * case["R"] * case["C"]
    params = 8 * case["N"] * case["C"]                       # weight and bias, or the weight and its statistics' gradients
    if case["what"] == "forward":
        return {"bytes": 2 * size * n + 8 * rows + params, "flops": 8 * n}
    return {"bytes": 3 * size * n + 8 * rows + 3 * params // 2, "flops": 14 * n}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["what"] in ("norm", "clip", "gather"):
        buffer, tensors, bound = _gradients(case, seed)
        total = torch.zeros(case["N"], dtype=torch.float64, device="cuda")
        for t in tensors:
            for i in range(case["N"]):
                total[i] += torch.linalg.vector_norm(t[i].double()) ** 2
        norms = total ** 0.5
        if case["what"] == "norm":
            return norms
        factor = (bound / norms).clamp_(max=1.0)
        if case["what"] == "clip":
            return torch.cat([(t.double() * factor[:, None]).reshape(-1) for t in tensors]), norms
        rows, at = torch.empty((case["N"], case["d"]), dtype=torch.float64, device="cuda"), 0
        for t in tensors:
            rows[:, at:at + t.shape[1]] = t
            at += t.shape[1]
        return rows.mul_(factor[:, None]), norms
    x, dy, models = _activations(case, seed)
    N, R, C = x.shape
    weight, bias = (v.double() for v in _columns(models, C))
    mean, rstd = (torch.empty((N, R), dtype=torch.float64, device="cuda") for _ in range(2))
    out = torch.empty((N, R, C), dtype=torch.float64, device="cuda")
    dweight, dbias = torch.empty_like(weight), torch.empty_like(bias)
    for i in range(N):                                       # a worker at a time
        v = x[i].double()
        var, mu = torch.var_mean(v, 1, correction=0, keepdim=True)
        mean[i], rstd[i] = mu[:, 0], (var[:, 0] + EPS) ** -0.5
        v = (v - mu) * rstd[i][:, None]
        if dy is None:
            out[i] = torch.addcmul(bias[i], v, weight[i])
            continue
        g = dy[i].double()
        dbias[i] = g.sum(0)
        dweight[i] = (g * v).sum(0)
        g *= weight[i]
        out[i] = (g - g.sum(1, keepdim=True) / C - v * ((g * v).sum(1, keepdim=True) / C)) * rstd[i][:, None]
    return (out, mean, rstd) if dy is None else (out, dweight, dbias)
