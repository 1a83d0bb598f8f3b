"""GPU tests of the router product's gradient where its precision or its ring of
staged weights can go wrong, against float64.

Tolerances (fixed before any GPU run), u = 2^-24:
* dx: dz enters as two bf16 terms rounded to nearest, off by at most 2^-17 of an
  element; n products are summed in fp32, n u of their sizes (2 n u for the two
  terms); one rounding to bf16, 2^-8 of the value.
* dW: dz enters whole, in three bf16 terms whose products with a bf16 are exact in fp32,
  so a single product is off by the two additions of its parts, 4 u with room to spare
  (without the third term by up to 2^-15); T products in 2 T u more.
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


@pytest.mark.parametrize("E", [1, 5, 16, 60, 100, 129, 250])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
def test_dx_of_an_infinite_router_weight(E, bad):
    """An infinite weight of the last expert shows in its column of dx (as an infinity or, since
    it is multiplied with both terms of dlogits, a NaN) and in no other."""
    banner("router dx inf", E, bad)
    T, H, c = 70, 192, 77
    g = torch.Generator(device=DEV)
    g.manual_seed(E)
    dz = torch.randn((T, E), generator=g, device=DEV)
    w = torch.randn((E, H), generator=g, device=DEV).bfloat16()
    w[E - 1, c] = bad
    dx, _, _, _ = moe.moe_router_grad(dz, torch.zeros((T, H), device=DEV).bfloat16(), w)
    assert not torch.isfinite(dx[:, c].float()).any()
    ok = torch.arange(H, device=DEV) != c
    check_dx(dx[:, ok], dz, w[:, ok])


# T, E, H: three column tiles or more a block (33 blocks of 128 rows share out the tiles
# among 512 blocks), of one, two and four pieces of W each; the last rows and, where H %
# 128 == 64, the last columns are not whole
@pytest.mark.parametrize("T,E,H", [(4099, 8, 7168), (4130, 64, 5184), (4099, 101, 7168), (4100, 128, 5184),
                                   (4129, 250, 5184), (4224, 256, 7168)])
def test_dx_of_many_column_tiles(T, E, H):
    banner("router dx tiles", T, E, H)
    g = torch.Generator(device=DEV)
    g.manual_seed(T + E)
    dz = torch.randn((T, E), generator=g, device=DEV) * torch.exp(torch.randn((T, 1), generator=g, device=DEV))
    x = torch.randn((T, H), generator=g, device=DEV).bfloat16()
    w = (torch.randn((E, H), generator=g, device=DEV) / H ** 0.5).bfloat16()
    room = torch.full((T + 130, H), 3.0, dtype=torch.bfloat16, device=DEV)
    dx, dw, db, _ = moe.moe_router_grad(dz, x, w, dx=room[:T])
    check_dx(dx, dz, w)
    assert (room[T:] == 3.0).all()
    a, b = dz.double(), x.double()
    assert ((dw.double() - a.t() @ b).abs() <= (2 * T + 8) * U * (a.abs().t() @ b.abs())).all()
    for _ in range(2):
        again = moe.moe_router_grad(dz, x, w)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)


@pytest.mark.parametrize("T,E,H", [(1, 1, 64), (16, 8, 128), (300, 100, 192), (4099, 256, 256), (2048, 255, 128)])
def test_dw_takes_all_bits_of_dlogits(T, E, H):
    """One token an expert has a gradient, with its low bits set, so every dW is a single
    product: it has all 24 bits of dlogits."""
    banner("router dw bits", T, E, H)
    r = np.random.default_rng(T + E)
    dz = np.zeros((T, E), np.float32)
    token = r.integers(0, T, E)
    odd = (r.integers(2 ** 23, 2 ** 24, E) | 0x7FFF).astype(np.float64) / 2 ** 23  # 15 low bits of 24
    dz[token, np.arange(E)] = odd * np.exp2(r.integers(-20, 20, E)) * r.choice([-1.0, 1.0], E)
    dz = torch.from_numpy(dz).to(DEV)
    x = torch.from_numpy(r.standard_normal((T, H))).to(DEV).bfloat16()
    w = torch.zeros((E, H), device=DEV).bfloat16()
    _, dw, db, _ = moe.moe_router_grad(dz, x, w, need_dx=False)
    want = dz.double().t() @ x.double()
    assert ((dw.double() - want).abs() <= 4 * U * want.abs()).all()
    assert torch.equal(db, dz.sum(0))


def test_dw_low_bits_add_up():
    """Columns of ones and gradients of one sign: what a dropped term of each would lose adds up."""
    banner("router dw sums")
    T, E, H = 64, 8, 64
    dz = torch.full((T, E), 1 + 2.0 ** -8 - 2.0 ** -23, device=DEV)
    x = torch.ones((T, H), device=DEV).bfloat16()
    _, dw, _, _ = moe.moe_router_grad(dz, x, torch.zeros((E, H), device=DEV).bfloat16(), need_dx=False)
    want = T * (1 + 2.0 ** -8 - 2.0 ** -23)
    assert ((dw.double() - want).abs() <= 2 * T * U * want).all()
