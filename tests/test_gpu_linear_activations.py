"""The activations by themselves, at the accuracy that is claimed for them: a layer of one weight 1 passes z through unrounded.

float32: a density whose exponent is off by 2^-23 of itself and some ulp of a polynomial: (16 + z^2) 2^-23 of the result, its negative tail
included.  SiLU: an exponential, a sum, a reciprocal, 8 x 2^-23 of the result.  Slopes: the same of each of their two terms.
Types of two bytes: the normal tail is off by 7.5e-8, everything else by 2^-21 of a term, and the result rounds."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES, TINY, U
pytestmark = pytest.mark.gpu
ULP = 2.0 ** -23


def points(T, reach):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    z = torch.cat([torch.linspace(-reach, reach, 40001, device="cuda"), torch.randn(40000, generator=g, device="cuda"),
                   torch.randn(4000, generator=g, device="cuda") * 1e-4, torch.zeros(1, device="cuda")])
    return z.to(T)[:, None].contiguous()


def terms(z, act):
    """The value, the slope and the sizes of the slope's terms in 64 bits.  (Phi by erfc: torch's ndtr takes 1 + erf on the GPU, which has no digits
    left of 3e-17 at z = -8.4.)"""
    if act == "gelu":
        Phi, phi = torch.erfc(-z / math.sqrt(2)) / 2, torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return z * Phi, Phi + z * phi, Phi + (z * phi).abs()
    s = 1 / (1 + torch.exp(-z))
    return z * s, s * (1 + z * torch.exp(-z) * s), s * (1 + z.abs())


@pytest.mark.parametrize("act,reach", [("gelu", 12.0), ("silu", 80.0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_accuracy(dtype, act, reach):
    z = points(dtype, reach)
    one = torch.ones((1, 1), dtype=dtype, device="cuda")
    y = vf.linear(z, one, activation=act)
    dx, _, _ = vf.linear_backward(torch.ones_like(z), z, one, z=z, activation=act, dweight=False, bias=False)
    Z = z.double()
    y64, s64, size = terms(Z, act)
    if dtype == torch.float32:
        rel = ((16 + Z * Z) if act == "gelu" else 8) * ULP
        bounds = rel * y64.abs(), (rel if act == "gelu" else 16 * ULP) * size
    else:
        e_y = 7.5e-8 * Z.abs() + 2.0 ** -21 * (y64.abs() + Z.abs() * torch.exp(-Z * Z / 4)) if act == "gelu" else 2.0 ** -23 * (4 + Z.abs()) * y64.abs()
        e_s = 7.5e-8 + 2.0 ** -21 * size if act == "gelu" else 2.0 ** -22 * (8 + Z.abs()) * size
        bounds = e_y + U[dtype] * (y64.abs() + e_y), e_s + U[dtype] * (s64.abs() + e_s)
    for got, want, tol, what in ((y, y64, bounds[0], "value"), (dx, s64, bounds[1], "slope")):
        off = (got.double() - want).abs() - tol - TINY[dtype]
        i = off.argmax().item()
        assert off.flatten()[i] <= 0, f"{what} at z = {Z.flatten()[i].item()}: {got.flatten()[i].item()}, not {want.flatten()[i].item()}"


@pytest.mark.parametrize("dtype", DTYPES)
def test_limits(dtype):
    """Infinite z, and finite ones beyond any exponential: the limits.  NaN stays NaN."""
    big = torch.finfo(dtype).max
    z = torch.tensor([[-math.inf], [-big], [-300.0], [300.0], [big], [math.inf], [math.nan]], dtype=dtype, device="cuda")
    one = torch.ones((1, 1), dtype=dtype, device="cuda")
    for act in ("relu", "gelu", "silu"):
        y = vf.linear(z, one, activation=act)[:, 0]
        dx = vf.linear_backward(torch.ones_like(z), z, one, z=z, activation=act, dweight=False, bias=False)[0][:, 0]
        assert not y[:3].any() and torch.equal(y[3:6], z[3:6, 0]) and torch.isnan(y[6])
        assert not dx[:3].any() and (dx[3:6] == 1).all() and torch.isnan(dx[6])
