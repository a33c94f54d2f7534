"""N simulated workers train a small normalised network with LIEC-SGD, each on data of its own, gradients clipped per worker.

Every worker's model is a row of `x`, its weights are views of that row.  The normalisation's weight gradients go straight into
tensors of [N, columns], the gradients of the products come from batched products, and liec_gather_grads clips them by their
global norm per worker on the way into the rows that LiecContext.iteration takes.

    python examples/clipped_training.py [--steps 200] [--workers 8] [--max-norm 1.0]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_11857_amd import LiecContext, liec_gather_grads, liec_layer_norm, liec_layer_norm_backward  # noqa: E402

FEATURES, HIDDEN, TARGETS = 48, 160, 10


class Workers:
    """Models of all workers as rows of `x`: out = relu(layer_norm(data @ first)) @ second."""

    SHAPES = (("first", (FEATURES, HIDDEN)), ("scale", (HIDDEN,)), ("shift", (HIDDEN,)), ("second", (HIDDEN, TARGETS)))

    def __init__(self, N: int, seed: int, device: str = "cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        start = {"first": torch.randn(FEATURES, HIDDEN, generator=gen, device=device) / FEATURES ** 0.5, "scale": torch.ones(HIDDEN, device=device),
                 "shift": torch.zeros(HIDDEN, device=device), "second": torch.randn(HIDDEN, TARGETS, generator=gen, device=device) / HIDDEN ** 0.5}
        self.N = N
        self.x = torch.cat([start[name].reshape(-1) for name, _ in self.SHAPES]).repeat(N, 1)
        self.d = self.x.shape[1]
        self.weights, at = {}, 0
        for name, shape in self.SHAPES:
            n = start[name].numel()
            self.weights[name] = self.x[:, at:at + n].view(N, *shape)
            at += n

    def loss_and_grads(self, data: torch.Tensor, target: torch.Tensor):
        """(loss of every worker, gradients as [N, ...] tensors in the order of SHAPES) on data [N, rows, FEATURES]."""
        w = self.weights
        h = torch.bmm(data, w["first"])
        z, mean, rstd = liec_layer_norm(h, w["scale"], w["shift"])
        a = z.clamp(min=0.0)
        off = torch.bmm(a, w["second"]) - target
        loss = off.square().mean((1, 2))
        dout = off * (2.0 / (off.shape[1] * off.shape[2]))
        dz = torch.bmm(dout, w["second"].transpose(1, 2).contiguous()) * (z > 0)
        dscale, dshift = torch.empty(self.N, HIDDEN, device=data.device), torch.empty(self.N, HIDDEN, device=data.device)
        dh = liec_layer_norm_backward(dz, h, mean, rstd, w["scale"], dx=dz, dweight=dscale, dbias=dshift)
        return loss, [torch.bmm(data.transpose(1, 2).contiguous(), dh), dscale, dshift, torch.bmm(a.transpose(1, 2).contiguous(), dout)]


def batches(N: int, rows: int, seed: int, device: str = "cuda"):
    """An endless sequence of (data, target): a fixed nonlinear map, seen by each worker on inputs of its own scale."""
    gen = torch.Generator(device=device).manual_seed(seed)
    hidden = torch.randn(FEATURES, TARGETS, generator=gen, device=device) / FEATURES ** 0.5
    scale = 0.5 + 1.5 * torch.rand(N, 1, 1, generator=gen, device=device)
    while True:
        data = torch.randn(N, rows, FEATURES, generator=gen, device=device) * scale
        yield data, torch.sin(2.0 * torch.matmul(data, hidden))


def train(steps: int = 200, N: int = 8, rows: int = 256, max_norm: float = 1.0, lr: float = 0.05, period: int = 32, seed: int = 1, report=None):
    """Mean loss of the workers at every step."""
    workers = Workers(N, seed)
    source = batches(N, rows, seed + 1)
    e = torch.zeros(workers.d, device="cuda")
    grads = torch.empty(N, workers.d, device="cuda")
    norms = torch.empty(N, device="cuda")
    losses = []
    with LiecContext(N, workers.d, "sign", "sign", lr=lr) as ctx:
        for t in range(steps):
            loss, tensors = workers.loss_and_grads(*next(source))
            liec_gather_grads(tensors, grads, max_norm, norms)
            ctx.iteration(t, period, grads, workers.x, e)
            losses.append(loss.mean())
            if report and t % report == 0:
                print(f"step {t:4d}  loss {float(losses[-1]):.4f}  gradient norms {float(norms.min()):.3f} .. {float(norms.max()):.3f}", flush=True)
    return torch.stack(losses).cpu()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args()
    train(a.steps, a.workers, max_norm=a.max_norm, report=20)
