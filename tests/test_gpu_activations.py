"""The linear layer's activations and their derivatives by themselves, u = 2^-24: a
product without terms leaves Z = bias, and the sums of D's one row are act'(Z).

GELU: Phi is off by at most 3 u, z Phi by |z| times that and a rounding of its own,
and the derivative by 3 u of Phi, 1 u of z times the density, whose exponent is
rounded, and 1 u of their sum.  Below zero Phi is off by 1e-5 of itself as well: the
exponent, up to 32 at z = -8, is rounded three times (48 u), and a sum of terms of 4
at most leaves 0.05 there (120 u)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0**-24


def _values():
    gen = torch.Generator().manual_seed(71)
    z = torch.cat([torch.linspace(-12, 12, 400001), torch.randn(200000, generator=gen),
                   torch.logspace(-30, 1, 1000), -torch.logspace(-30, 1, 1000)])
    return z.cuda()


def _forward(z, activation):
    import paper_2507_23387_amd as sgc

    n = z.numel()
    empty = torch.zeros((1, 0), device="cuda"), torch.zeros((0, n), device="cuda")
    return sgc.linear(*empty, bias=z, activation=activation)[0]


def _derivative(z, activation):
    import paper_2507_23387_amd as sgc

    n = z.numel()
    X, W = torch.zeros((1, 1), device="cuda"), torch.zeros((1, n), device="cuda")
    return sgc.linear_backward(torch.ones((1, n), device="cuda"), X, W, z[None], activation,
                               need=("db",))[2]


def _phi(z):
    # Not torch.special.ndtr, which is 1 + erf in the tail: 4e-2 of itself off at z = -8.
    return 0.5 * torch.special.erfc(-z / math.sqrt(2))


def test_gelu(gpu):
    z = _values()
    z64 = z.double()
    want = z64 * _phi(z64)
    error = (_forward(z, "gelu").double() - want).abs()
    worst = (error / (3 * U * z64.abs() + U * want.abs() + 2.0**-126)).max().item()
    assert worst <= 1, f"{worst:.3f} of the bound"
    tail = (z < 0) & (z >= -8)
    worst = (error[tail] / want[tail].abs()).max().item()
    assert worst <= 1e-5, f"{worst:.2e} of itself below zero"


def test_gelu_derivative(gpu):
    z = _values()
    z64 = z.double()
    density = torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    want = _phi(z64) + z64 * density
    worst = ((_derivative(z, "gelu").double() - want).abs() / (5 * U)).max().item()
    assert worst <= 1, f"{worst:.3f} of the bound"


@pytest.mark.parametrize("activation", ["relu", "gelu", "gelu_tanh", "silu"])
def test_far_from_zero(gpu, activation):
    """z itself and 1 above, 0 below, up to the largest float."""
    z = torch.tensor([50.0, 1e4, 1e13, 1e19, 2e19, 1e30, 3.4e38], device="cuda")
    z = torch.cat([z, -z])
    positive = z > 0
    # exp(50) is 5e21: sigmoid and Phi are 1 to the last bit above zero, and below 50 exp(-50)
    # is under 1e-19.
    y = _forward(z, activation)
    assert torch.equal(y[positive], z[positive]) and torch.all(y[~positive].abs() <= 1e-19)
    assert torch.all((_derivative(z, activation) - positive.float()).abs() <= 1e-19)
