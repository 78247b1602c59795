"""Plain 64-bit forms of the feed-forward operators and the bounds that their kernels are held to.

Bounds follow from the arithmetic.  u = 2^-24 is the rounding of a float32 operation, 2^-8 that of a result stored in bf16.
A sum of n products accumulated in float32 in any order is within about n u of its terms' absolute sum; the kernels add in
blocks of at least 32, so n / 32 steps and the blocks' own few are allowed."""

import math

import torch

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def store(dtype):
    """Relative rounding of a stored result (1 % more than half a unit, for the float32 value in front of it)."""
    return 2.0 ** -8 * 1.01 if dtype == torch.bfloat16 else 2.0 ** -24 * 1.01


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def act(z, name):
    if name == "silu":
        return z * torch.special.expit(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    return torch.relu(z) if name == "relu" else z


def slope(z, name):
    if name == "silu":
        s = torch.special.expit(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return (z > 0).double() if name == "relu" else torch.ones_like(z)


def assert_within(got, want, bound, what=""):
    """|got - want| <= bound elementwise (float64 tensors on the CPU; NaN fails)."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        i = int(torch.nonzero(bad.reshape(-1))[0])
        raise AssertionError("%s: %d of %d outside the bound, first at %d: got %r want %r bound %r" % (
            what, int(bad.sum()), bad.numel(), i, got.reshape(-1)[i].item(), want.reshape(-1)[i].item(),
            torch.as_tensor(bound).expand_as(want).reshape(-1)[i].item()))


def sum_bound(n, f32_operands=False):
    """Rounding of a contraction over n, relative to the absolute sum of its terms (six products a term where float32 operands
    are taken in pieces, and what is dropped of them)."""
    steps = n / 32 * (6 if f32_operands else 1) + 24
    return (steps + (4 if f32_operands else 0)) * 2 * U


ACT_LIP = 1.13  # largest slope of the activations
ACT_REL = 16 * U  # of an activation's own evaluation: a fast exponential, a reciprocal, an error function
