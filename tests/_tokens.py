"""Helpers shared by the tests of the token operators."""
import torch

U = 2.0 ** -24  # unit roundoff of fp32
BF, F, D64 = torch.bfloat16, torch.float32, torch.float64


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def full(shape, dtype=F, value=77.0):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def count_of(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def rounding(dtype, v):
    """Half a step of the output's type."""
    return torch.finfo(dtype).eps / 2 * v.abs()


def within(got, ref, tol, what):
    got = got.to(D64)
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float(((got - ref).abs() - tol).max()):.3e} over its bound")


def shifted(t):
    """A copy whose first element lies one past a 16-byte boundary."""
    s = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
    return s.copy_(t)
