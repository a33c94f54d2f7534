"""Shared pieces of the tests of the operators around a backward pass: types, unit roundoffs and seeded inputs."""
import torch

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U32 = 2.0 ** -24                                             # unit roundoffs: half the spacing of numbers just above 1
U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}    # smallest subnormal numbers


def generator(seed, device="cuda:0"):
    return torch.Generator(device=device).manual_seed(seed)


def assert_within(got, want, bound, what):
    """|got - want| <= bound element by element, in 64 bits."""
    err = (got.double() - want).abs()
    bad = ~(err <= bound)                                    # NaN counts as bad
    if bad.any():
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, first at {i}: got {got.reshape(-1)[i].item()!r}, "
                             f"want {want.reshape(-1)[i].item()!r}, bound {torch.broadcast_to(bound, err.shape).reshape(-1)[i].item()!r}")
