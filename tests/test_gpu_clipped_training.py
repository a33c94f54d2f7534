"""The example that runs normalisation, its gradients, clipping and the compressed step together: its gradients against
automatic differentiation of the same network in 64 bits, and the training itself."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402

pytestmark = GPU_MARKS


@pytest.fixture(scope="module")
def example():
    import importlib.util

    spec = importlib.util.spec_from_file_location("clipped_training", os.path.join(ROOT, "examples", "clipped_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_and_clipped_rows(example):
    from paper_2402_11857_amd import liec_gather_grads

    say("case example, gradients of 5 workers")
    N = 5
    workers = example.Workers(N, seed=3)
    workers.x += 0.05 * torch.randn(workers.x.shape, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV)     # models that differ
    data, target = next(example.batches(N, 33, seed=5))
    loss, tensors = workers.loss_and_grads(data, target)
    # the same in 64 bits, worker by worker, from the flat models
    x = workers.x.double().requires_grad_()
    total, losses = 0.0, []
    for i in range(N):
        at, w = 0, {}
        for name, shape in workers.SHAPES:
            n = torch.Size(shape).numel()
            w[name] = x[i, at:at + n].view(shape)
            at += n
        h = data[i].double() @ w["first"]
        h = (h - h.mean(1, keepdim=True)) / torch.sqrt(h.var(1, keepdim=True, correction=0) + 1e-5) * w["scale"] + w["shift"]
        losses.append((torch.relu(h) @ w["second"] - target[i].double()).square().mean())
        total = total + losses[-1]
    total.backward()
    want = x.grad
    # fp32 products over up to 256 terms and the normalisation's own rounding: 2e-5 of a worker's largest gradient
    size = want.abs().amax(1, keepdim=True)
    rows = torch.empty(N, workers.d, device=DEV)
    norms = torch.empty(N, device=DEV)
    liec_gather_grads(tensors, rows)
    assert torch.allclose(loss.double(), torch.stack(losses).detach(), rtol=1e-5, atol=0)
    assert float(((rows.double() - want).abs() / size).max()) < 2e-5
    norm = want.norm(dim=1)
    bound = float(norm.median())
    liec_gather_grads(tensors, rows, bound, norms)
    assert float((norms.double() / norm - 1).abs().max()) < 2e-5
    clipped = want * torch.clamp(bound / norm, max=1.0)[:, None]
    assert float(((rows.double() - clipped).abs() / size).max()) < 2e-5


def test_training_reduces_the_loss_and_is_reproducible(example):
    say("case example, 150 steps of 8 workers, twice")
    first = example.train(steps=150)
    assert first.isfinite().all()
    assert float(first[-10:].mean()) < 0.8 * float(first[:10].mean())
    assert torch.equal(first, example.train(steps=150))
