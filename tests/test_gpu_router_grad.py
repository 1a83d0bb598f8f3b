"""GPU tests of the router product's gradient where its precision or its ring of
staged weights can go wrong, against float64.

Tolerances (fixed before any GPU run), u = 2^-24:
* dx: dz enters as two bf16 terms rounded to nearest, off by at most 2^-17 of an
  element; n products are summed in fp32, n u of their sizes (2 n u for the two
  terms); one rounding to bf16, 2^-8 of the value with both sides of a boundary.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


def check_dx(dx, dz, w):
    a, c = dz.double(), w.double()
    want, size = a @ c, a.abs() @ c.abs()
    tol = (2.0 ** -17 + 2 * dz.shape[1] * U) * size + 2.0 ** -8 * want.abs()
    err = (dx.double() - want).abs()
    assert (err <= tol).all(), float((err / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("T,E,H", [(5, 8, 64), (200, 7, 192), (33, 12, 1024)])
def test_dx_of_rows_that_cancel(T, E, H):
    """dz rows whose sum is small beside their elements and router rows that are alike:
    what is left of dx is as small as what dz loses when its terms are cut off instead
    of rounded (2^-15 of every positive element)."""
    banner("router dx cancel", T, E, H)
    r = np.random.default_rng(T)
    dz = np.full((T, E), 1 + 2.0 ** -8 + 2.0 ** -15 - 2.0 ** -23)
    dz[:, 0] = -(E - 1) * (1 + 2.0 ** -8)
    dz *= np.exp2(r.integers(-30, 30, (T, 1)))
    dz = torch.from_numpy(np.take_along_axis(dz, r.permuted(np.tile(np.arange(E), (T, 1)), axis=1), 1)).float().to(DEV)
    w = torch.ones((E, H), device=DEV).bfloat16() * torch.from_numpy(np.exp2(r.integers(-3, 3, (1, H)))).to(DEV).bfloat16()
    dx, _, _, _ = moe.moe_router_grad(dz, torch.zeros((T, H), device=DEV).bfloat16(), w)
    check_dx(dx, dz, w)


def test_dx_of_the_largest_and_smallest_gradients():
    """Values that bf16 would round up to infinity stay finite; denormals do no harm."""
    banner("router dx extremes")
    T, E, H = 4, 8, 64
    dz = torch.zeros((T, E), device=DEV)
    dz[0, 3], dz[1, 7] = torch.finfo(torch.float32).max, -3.4e38
    dz[2, 0], dz[2, 1] = 1e-38, -3e-39
    w = torch.full((E, H), 0.5, device=DEV).bfloat16()
    dx, _, _, _ = moe.moe_router_grad(dz, torch.zeros((T, H), device=DEV).bfloat16(), w)
    assert torch.isfinite(dx.float()).all()
    want = dz.double() @ w.double()
    assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-38).all()
