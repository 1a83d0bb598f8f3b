"""GPU tests of the training calls at their largest token counts, where an index past 31
bits would show in the counts and at the ends of the outputs.

Tolerances (fixed before any GPU run), u = 2^-24: sums of terms of one sign in fp32
within a block, at most 64 additions a lane and 16 between lanes, the blocks in fp64:
relative 128 u, with exp and log to 2 ulp.
"""
import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,seq", [(2 ** 31 - 256, 0), (2 ** 23 - 1, 1)])
def test_balance_at_the_block_limit(T, seq):
    """Two experts, every token with logits (0, log 3); the first of them from token 5 on."""
    banner("balance limit", T, seq)
    E, G = 2, T // seq if seq else 1
    z = torch.zeros((T, E), device=DEV)
    z[:, 1] = 1.0986122886681098
    ids = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    ids[:5] = 1
    loss, counts, live, ws = moe.moe_balance_loss(z, ids, seq_len=seq)
    lse = 2 * 0.6931471805599453
    want = [2 * (0.25 * (T - 5) + 0.75 * 5) / T, lse * lse]
    assert all(abs(float(a) - b) <= 128 * U * b for a, b in zip(loss, want)), (loss, want)
    assert live[:G].sum() == T and live[-2:].tolist() == [T, G] and not ws[:256].any()
    if seq:
        assert (counts[:5] == torch.tensor([0, 1], device=DEV)).all() and (counts[5:] == torch.tensor([1, 0], device=DEV)).all()
    else:
        assert counts.tolist() == [[T - 5, 5]]
    del ws
    d = moe.moe_gate_backward(z, ids, counts, live, torch.tensor([0.0, float(T)], device=DEV), seq_len=seq)
    want = 2 * lse * torch.tensor([0.25, 0.75], device=DEV)
    for at in (slice(0, 300), slice(T // 2, T // 2 + 300), slice(T - 300, T)):
        assert ((d[at] - want).abs() <= 128 * U * want).all()


@pytest.mark.parametrize("T", [2 ** 25, 2 ** 25 + 1, 2 ** 26 + 5, 2 ** 31 - 1])
def test_combine_backward_of_many_tokens(T):
    """All remote but some tokens at the ends and around every 2^25-th: dw = <dout, y>."""
    banner("combine limit", T)
    H = 4
    at = sorted({a for b in range(0, T + 2 ** 25, 2 ** 25) for a in (b - 1, b, b + 3) if 0 <= a < T} | {T - 4, T - 1})
    n = len(at)
    r = torch.Generator(device=DEV)
    r.manual_seed(T)
    where = torch.tensor(at, device=DEV)
    y = torch.randn((n, H), generator=r, device=DEV)
    do = torch.randn((n, H), generator=r, device=DEV)
    w = torch.rand(n, generator=r, device=DEV)
    order = torch.randperm(n, generator=r, device=DEV)
    dout = torch.ones((T, H), device=DEV)
    dout[where] = do
    dest = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    dest[where] = order.int()
    weights = torch.zeros((T, 1), device=DEV)
    weights[where, 0] = w
    dw = torch.full((T, 1), 7.0, device=DEV)
    _, dy = moe.moe_combine_backward(dout, y, weights, dest, dweights=dw)
    want, size = (do.double() * y[order].double()).sum(1), (do * y[order]).abs().sum(1)
    assert ((dw[where, 0].double() - want).abs() <= 4 * U * size).all()
    assert torch.equal(dy[order], w.unsqueeze(1) * do)
    dw[where] = 0.0
    assert not dw.any()


@pytest.mark.parametrize("T,E,H,dtype", [(2 ** 31 - 1, 1, 8, torch.float32), (2 ** 31 - 3, 1, 8, torch.float32),
                                         (2 ** 26 + 33, 3, 64, torch.bfloat16)])
def test_router_grad_of_many_tokens(T, E, H, dtype):
    """dlogits are zero but for a few tokens, at the ends and in the middle of the ranges."""
    banner("router limit", T, E, H, dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    where = torch.tensor([0, 1, 31, T // 64, T // 2, T - 300, T - 33, T - 5, T - 2, T - 1], device=DEV)
    n = where.numel()
    dz = torch.zeros((T, E), device=DEV)
    dz[where] = torch.randn((n, E), generator=g, device=DEV)
    x = torch.ones((T, H), dtype=dtype, device=DEV)
    x[where] = torch.randn((n, H), generator=g, device=DEV).to(dtype)
    w = torch.randn((E, H), generator=g, device=DEV).to(dtype)
    bf16 = dtype == torch.bfloat16
    dx, dw, db, _ = moe.moe_router_grad(dz, x, w, need_dx=bf16)
    a, b = dz[where].double(), x[where].double()
    assert ((dw.double() - a.t() @ b).abs() <= 3 * n * U * (a.abs().t() @ b.abs())).all()
    assert ((db.double() - a.sum(0)).abs() <= n * U * a.abs().sum(0)).all()
    if bf16:
        want, size = a @ w.double(), a.abs() @ w.abs().double()
        assert ((dx[where].double() - want).abs() <= (2.0 ** -17 + 2 * E * U) * size + 2.0 ** -8 * want.abs()).all()
        dx[where] = 0.0
        assert not dx.any()
