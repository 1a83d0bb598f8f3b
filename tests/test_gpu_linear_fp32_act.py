"""GPU tests of the fp32 product's activations and their slopes, which are to be as exact as
fp32 makes them at any size of the pre-activation.

x is a row of zeros but for a 1, so z is a weight, exactly. Bounds, u = 2^-24 (half a step of
fp32):
* silu: an exponential (2 u), a sum, a product and a quotient (u each), 5 u of the value;
* its slope q + z q (1 - q) = q (1 + z r): q and r = 1 - q by e / (1 + e) and 1 / (1 + e), off by 5 u at
  most each; z r by 6 u of itself, so |z| q r by 11 u; sum and product round once each: 11 u of
  q + |z| q r and 2 u of the value;
* gelu: z Phi(z); Phi from an error function of -z / sqrt 2, whose rounding (1.5 u of it) moves
  the value by z^2 times that where z < 0, below 2 z^2 u in all; the function's own 16 ulp at most, 32 u;
  two products. (36 + 2 z^2) u of the value;
* its slope Phi + z phi: phi's exponent rounds z^2 twice, z^2 u of phi, 6 u for the exponential and the
  products: (40 + 2 z^2) u of Phi + |z| phi;
and what underflows: 2^-126 of |z| + 1.
"""
import math

import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def points():
    z = torch.cat([torch.linspace(-110, 110, 4401), torch.linspace(-16, 16, 4001), torch.logspace(-30, 0, 200), -torch.logspace(-30, 0, 200),
                   torch.tensor([0.0, -0.0, 3e38, -3e38, 1e20, -1e20, -87.4, -88.0, -88.8, -89.5, -103.0])]).float()
    return torch.cat([z, z.new_zeros(-z.numel() % 8)]).to(DEV)


def exact(z, act):
    """The value, the slope and the size of the slope's terms, in 64 bits."""
    z = z.double()
    if act == "silu":
        q, r = torch.sigmoid(z), torch.sigmoid(-z)
        return z * q, q + z * q * r, q + (z * q * r).abs()
    q = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    p = z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    p = torch.where(torch.isfinite(p), p, torch.zeros_like(p))
    return z * q, q + p, q + p.abs()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_values_and_slopes(act):
    print("CASE linear fp32 activation", act, flush=True)
    z = points()
    N, K = z.numel(), 8
    x = torch.zeros((1, K), device=DEV)
    x[0, 0] = 1.0
    w = torch.zeros((N, K), device=DEV)
    w[:, 0] = z
    kept = torch.empty((1, N), device=DEV)
    y = moe.moe_linear(x, w, act=act, z=kept)[0]
    assert torch.equal(kept[0], z)
    value, slope, size = exact(z, act)
    a = z.double().abs()
    tiny = 2.0 ** -126 * (a + 1)
    tol = (5 * U if act == "silu" else (36 + 2 * a * a) * U) * value.abs() + tiny
    err = (y.double() - value).abs()
    assert (err <= tol).all(), (float((err / tol).max()), z[err > tol][:8].tolist())
    dz = moe.moe_linear_backward(torch.ones((1, N), device=DEV), x, w, z=kept, act=act, need_dx=False, need_dw=False, need_dbias=False)[3][0]
    tol = (11 * U * size + 2 * U * slope.abs() if act == "silu" else (40 + 2 * a * a) * U * size) + tiny
    err = (dz.double() - slope).abs()
    assert (err <= tol).all(), (float((err / tol).max()), z[err > tol][:8].tolist())
    # the gate's gradient takes the same values
    dmul = moe.moe_linear_backward(torch.ones((1, N), device=DEV), x, w, z=kept, act=act, mul=torch.ones((1, N), device=DEV), need_dx=False,
                                   need_dw=False, need_dbias=False)[4][0]
    assert torch.equal(dmul, y)
