"""Shared pieces of the tests of the operators on activations: seeded inputs and the checkpoint's definition in 64 bits."""
import torch

from _gpu import DEV
from _train import DTYPES, generator


def activations(shape, dtype, seed, offset=0.5):
    gen = generator(seed)
    C = shape[-1]
    x = torch.randn(shape, generator=gen, device=DEV) * (0.25 + 2 * torch.rand(C, generator=gen, device=DEV)) + offset * torch.randn(C, generator=gen, device=DEV)
    return x.to(DTYPES[dtype])


def power(k):
    """2^k in 64 bits, exactly."""
    return (k.long() + 1023 << 52).view(torch.float64)


def expected_checkpoint(x):
    """(values, exponents) of a checkpoint of x from the definition, by search from the smallest exponent upwards in 64 bits."""
    C = x.shape[-1]
    v = torch.nn.functional.pad(x.double(), (0, -C % 32)).unflatten(-1, (-1, 32))
    largest = v.abs().amax(-1)
    bad = ~torch.isfinite(v).all(-1)
    _, e = torch.frexp(torch.where(bad, torch.ones_like(largest), largest))
    k = torch.where(largest > 0, torch.clamp(e - 8, min=-126), -126)      # too small, or the smallest
    for _ in range(3):
        k = torch.where(largest >= 127.5 * power(k), k + 1, k)
    k = torch.where(bad, torch.zeros_like(k), k).clamp(max=121)          # 127 * 2^121 is the largest number
    q = (v / power(k)[..., None]).round().clamp(-127, 127)
    q = torch.where(bad[..., None], torch.zeros_like(q), q)
    return q.flatten(-2)[..., :C].to(torch.int8), torch.where(bad, torch.full_like(k, 255), k + 127).to(torch.uint8)


def value(saved, dtype=torch.float64):
    """What a checkpoint stands for, in 64 bits."""
    q, s = saved
    scale = torch.where(s == 255, torch.full(s.shape, float("nan"), dtype=torch.float64, device=s.device), power(s.long() - 127))
    return (q.double() * scale.repeat_interleave(32, -1)[..., :q.shape[-1]]).to(dtype)
