"""GPU tests of the dense products' large tiles, splits and shared launches: every part of
the epilogue, rows cut from the last round, the bias' sums from dw's tiles, both types of dw,
values that are not finite.

Integers: sums stay below 2^24, so results are exact in fp32 and rounded once. Activations:
u = 2^-24; a sum of n products is off by (n + 2) u of the sum of their sizes, the bias
included; silu's and gelu's slopes are below 1.13; their own errors are (8 + 2 |z|) u |z| (an
exponential of a rounded argument, a reciprocal, three products) and (16 + z^2) u |z|; the
gate multiplies that, gate and residual round once each, the result is rounded by 2^-8.
"""
import math

import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def ints(g, *shape, lo=-3, hi=4, dtype=BF):
    return torch.randint(lo, hi, shape, generator=g, device=DEV).to(dtype)


def normal(g, *shape, dtype=BF, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


# On 256 CUs: 256 x 256 tiles with no, one and three whole chunks; the same with the last rows
# apart; with the reduction in ranges; 128 x 128 tiles for at most a CU each and for more; 64 x 64
# tiles in ranges
FORWARD = [(3601, 3592, 40), (3601, 3592, 72), (3601, 3592, 200), (2422, 14336, 1032), (1032, 2424, 14336), (1800, 2056, 520),
           (2050, 2056, 4104), (600, 1032, 4104), (300, 256, 4096)]


@pytest.mark.parametrize("M,N,K", FORWARD)
def test_epilogue_of_integers(M, N, K):
    print("CASE linear large epilogue ints", M, N, K, flush=True)
    g = gen(M + N + K)
    x, w = ints(g, M, K), ints(g, N, K)
    b, m, r = ints(g, N, lo=-40, hi=41, dtype=torch.float32), ints(g, M, N), ints(g, M, N)
    plain = x.double() @ w.double().t()
    for bias, mul, res, act in ((b, m, r, "none"), (b, None, None, "relu"), (None, m, None, "relu"), (b, None, r, "none"),
                                (None, m, r, "relu")):
        zz = plain if bias is None else plain + bias.double()
        z = torch.full((M, N), 9.0, device=DEV, dtype=BF)
        y = moe.moe_linear(x, w, bias=bias, mul=mul, residual=res, act=act, z=z)
        want = zz.clamp(min=0) if act == "relu" else zz
        if mul is not None:
            want = want * mul.double()
        if res is not None:
            want = want + res.double()
        assert torch.equal(z, zz.to(BF))
        assert torch.equal(y, want.to(BF)), (bias is None, mul is None, res is None, act)
        assert torch.equal(moe.moe_linear(x, w, bias=bias, mul=mul, residual=res, act=act), y)  # without z
    # in place of the gate and of the residual
    y = moe.moe_linear(x, w, bias=b, mul=m, residual=r)
    for name in ("mul", "residual"):
        t = (m if name == "mul" else r).clone()
        kw = {"mul": m, "residual": r, name: t}
        assert torch.equal(moe.moe_linear(x, w, bias=b, out=t, **kw), y)


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,N,K", [(3601, 3592, 200), (2422, 14336, 1032), (1032, 2424, 14336), (1800, 2056, 520)])
def test_activations(M, N, K, act):
    print("CASE linear large activations", M, N, K, act, flush=True)
    g = gen(K)
    x, w = normal(g, M, K), normal(g, N, K, scale=2 / K ** 0.5)
    b, m, r = normal(g, N, dtype=torch.float32), normal(g, M, N), normal(g, M, N)
    z64 = x.double() @ w.double().t() + b.double()
    dz = (K + 2) * U * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    a = z64.abs()
    own = (8 + 2 * a) * U * a if act == "silu" else (16 + a * a) * U * a
    z = torch.empty((M, N), dtype=BF, device=DEV)
    for mul, res in ((None, None), (m, r)):
        y = moe.moe_linear(x, w, bias=b, act=act, mul=mul, residual=res, z=z)
        assert ((z.double() - z64).abs() <= dz + 2.0 ** -8 * z64.abs()).all()
        want = act64(z64, act)
        tol = 1.13 * dz + own + 1e-37
        if mul is not None:
            want = want * mul.double()
            tol = tol * mul.double().abs() + U * want.abs()
            want = want + res.double()
            tol = tol + U * want.abs()
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
        assert ((y.double() - want).abs() <= tol).all()


# On 256 CUs, dw by 256 x 256 tiles that also sum dy: the tiles' column j of J sums the chunks j,
# j + J, ...: 23 chunks and a part in 6 columns, 32 and a part in 15, 32 and a part in 17, 4 and a
# part in 33; then dx in ranges, dw with its last rows apart, 128 x 128 tiles, and both gradients in one
# launch of either tile
BACKWARD = [(1500, 7168, 1288), (2100, 3592, 3608), (2050, 2056, 4104), (300, 1032, 8200), (2422, 14336, 1032), (1032, 2424, 14336),
            (4100, 1032, 4104), (9001, 768, 1000), (1800, 2056, 520), (1200, 1288, 264)]


@pytest.mark.parametrize("M,N,K", BACKWARD)
@pytest.mark.parametrize("dw_dtype", [torch.float32, BF])
def test_gradients_of_integers(M, N, K, dw_dtype):
    print("CASE linear large backward ints", M, N, K, dw_dtype, flush=True)
    g = gen(M + N + K)
    # dbias adds up to 9001 values of up to 9
    x, w, dy = ints(g, M, K), ints(g, N, K), ints(g, M, N)
    full = dy.double().t() @ x.double()
    dx, dw, db, dz, _ = moe.moe_linear_backward(dy, x, w, dw_dtype=dw_dtype)
    assert dz is dy and dw.dtype == dw_dtype
    assert torch.equal(db, dy.double().sum(0).float())
    assert torch.equal(dx, (dy.double() @ w.double()).to(BF)) and torch.equal(dw, full.to(dw_dtype))
    # each by itself
    assert torch.equal(moe.moe_linear_backward(dy, x, w, need_dx=False, need_dw=False)[2], db)
    assert torch.equal(moe.moe_linear_backward(dy, x, w, need_dx=False, need_dbias=False, dw_dtype=dw_dtype)[1], dw)
    assert torch.equal(moe.moe_linear_backward(dy, x, w, need_dw=False, need_dbias=False)[0], dx)
    # an activation and a gate
    z, m = ints(g, M, N), ints(g, M, N)
    dx, dw, db, dz, dmul = moe.moe_linear_backward(dy, x, w, z=z, mul=m, act="relu", dw_dtype=dw_dtype)
    want = dy.double() * m.double() * (z > 0)
    assert torch.equal(dz, want.to(BF)) and torch.equal(dmul, (dy.double() * z.double().clamp(min=0)).to(BF))
    assert torch.equal(db, want.sum(0).float())
    assert torch.equal(dx, (want @ w.double()).to(BF)) and torch.equal(dw, (want.t() @ x.double()).to(dw_dtype))


# few rows by 8 and by 16 columns a block, two blocks of 16 rows; 64 x 64 tiles in ranges; 128 x 128 tiles; large
# ones with the last rows apart and in ranges
@pytest.mark.parametrize("M,N,K", [(8, 264, 200), (5, 136, 1032), (8, 6000, 72), (16, 136, 200), (31, 264, 1000), (300, 256, 4096),
                                   (1800, 2056, 520), (3601, 3592, 72), (2422, 14336, 1032), (1032, 2424, 14336)])
def test_values_that_are_not_finite_stay_in_their_row_or_column(M, N, K):
    print("CASE linear large NaN", M, N, K, flush=True)
    g = gen(M)
    x, w = ints(g, M, K), ints(g, N, K)
    want = moe.moe_linear(x, w)
    x2, w2 = x.clone(), w.clone()
    rows, cols = sorted({0, M // 2, M - 1}), sorted({1, N // 2, N - 1})
    x2[0, K // 2 + 1], x2[M // 2, K - 1], x2[M - 1, 0] = NAN, INF, NAN
    for v, c, at in zip((NAN, -INF, NAN), (1, N // 2, N - 1), (K - 3, 1, K // 2)):
        w2[c, at] = v
    y = moe.moe_linear(x2, w)
    keep = torch.ones(M, dtype=torch.bool, device=DEV)
    keep[rows] = False
    assert torch.equal(y[keep], want[keep])
    assert torch.isnan(y[0]).all() and torch.isnan(y[M - 1]).all() and not torch.isfinite(y[M // 2]).any()
    y = moe.moe_linear(x, w2)
    keep = torch.ones(N, dtype=torch.bool, device=DEV)
    keep[cols] = False
    assert torch.equal(y[:, keep], want[:, keep])
    assert torch.isnan(y[:, 1]).all() and torch.isnan(y[:, N - 1]).all()
    # an infinity times a zero is NaN, times another value infinite
    assert torch.equal(torch.isnan(y[:, N // 2]), x[:, 1] == 0) and not torch.isfinite(y[:, N // 2]).any()


# both gradients in one launch of 64 x 64 and of 128 x 128 tiles; in ranges; large tiles; large ones that sum dy
@pytest.mark.parametrize("M,N,K", [(65, 264, 1000), (700, 520, 2056), (40, 3592, 3608), (2422, 14336, 1032), (1032, 2424, 14336),
                                   (1500, 7168, 1288)])
def test_gradients_that_are_not_finite_stay_in_their_row_or_column(M, N, K):
    print("CASE linear large backward NaN", M, N, K, flush=True)
    g = gen(N)
    x, w, dy = ints(g, M, K), ints(g, N, K), ints(g, M, N)
    dx, dw, db, _, _ = moe.moe_linear_backward(dy, x, w)
    bad = dy.clone()
    bad[M - 1, N - 1] = NAN
    bad[M // 2, 3] = INF
    dx2, dw2, db2, _, _ = moe.moe_linear_backward(bad, x, w)
    rows, cols = torch.ones(M, dtype=torch.bool, device=DEV), torch.ones(N, dtype=torch.bool, device=DEV)
    rows[[M - 1, M // 2]] = False
    cols[[N - 1, 3]] = False
    assert torch.equal(dx2[rows], dx[rows]) and torch.isnan(dx2[M - 1]).all() and not torch.isfinite(dx2[M // 2]).any()
    assert torch.equal(dw2[cols], dw[cols]) and torch.isnan(dw2[N - 1]).all() and not torch.isfinite(dw2[3]).any()
    assert torch.equal(db2[cols], db[cols]) and torch.isnan(db2[N - 1]) and db2[3] == INF
    # of the weights to a column of dx, of the tokens to a column of dw
    w2, x2 = w.clone(), x.clone()
    w2[N - 1, K - 1] = NAN
    x2[M - 1, 2] = NAN
    dx2, dw2, _, _, _ = moe.moe_linear_backward(dy, x2, w2, need_dbias=False)
    keep = torch.arange(K, device=DEV)
    assert torch.equal(dx2[:, keep != K - 1], dx[:, keep != K - 1]) and torch.isnan(dx2[:, K - 1]).all()
    assert torch.equal(dw2[:, keep != 2], dw[:, keep != 2]) and torch.isnan(dw2[:, 2]).all()


@pytest.mark.parametrize("M,N,K", [(1500, 7168, 1288), (2422, 14336, 1032)])
def test_graph_beside_eager_calls(M, N, K):
    """A captured step, replayed with other inputs and eager calls between, repeats their bits."""
    print("CASE linear large graph", M, N, K, flush=True)
    g = gen(5)
    x, w, dy, b = normal(g, M, K), normal(g, N, K, scale=1 / K ** 0.5), normal(g, M, N), normal(g, N, dtype=torch.float32)
    def buffers():
        return dict(ws=torch.empty(moe.linear_ws_bytes(M, N, K, BF), dtype=torch.uint8, device=DEV),
                    wb=torch.empty(moe.linear_backward_ws_bytes(M, N, K, BF), dtype=torch.uint8, device=DEV),
                    y=torch.empty((M, N), dtype=BF, device=DEV), dx=torch.empty((M, K), dtype=BF, device=DEV),
                    dw=torch.empty((N, K), device=DEV), db=torch.empty(N, device=DEV))

    def step(t):
        moe.moe_linear(x, w, bias=b, act="silu", mul=dy, out=t["y"], ws=t["ws"])
        moe.moe_linear_backward(dy, x, w, dx=t["dx"], dw=t["dw"], dbias=t["db"], ws=t["wb"])

    one, two = buffers(), buffers()
    step(one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(one)
    for _ in range(3):
        x.copy_(normal(g, M, K))
        dy.copy_(normal(g, M, N))
        for t in one.values():
            t.fill_(3)
        graph.replay()
        step(two)
        torch.cuda.synchronize()
        assert all(torch.equal(one[n], two[n]) for n in ("y", "dx", "dw", "db"))
