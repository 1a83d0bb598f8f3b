"""GPU tests of the dense products and their gradients against float64.

Tolerances (fixed before any GPU run), u = 2^-24, h = 2^-8 (bf16) or u (fp32), the rounding of
a value:
* products of integers below 2^24 in sum are exact: outputs without an activation are
  compared bit for bit with the rounded exact value;
* a sum of n products is off by (n + 2) u of the sum of their sizes, S, bias included;
* an activation passes an error on with its slope, below 1.13, and adds its own: an
  exponential (2 ulp and u |z| of its argument), a reciprocal (1 ulp), three products: (8 + 2 |z|)
  u of |z| for silu; gelu's erfc: 16 u of the value's bound |z| and z^2 u from its argument;
  of their slopes (below 1.13, terms of |z| q (1 - q)): the same times (1 + |z|);
* mul multiplies that; residual and the roundings add u each; then one rounding h of the
  result;
* dx and dw are compared with the products of the dz that the call left.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF = torch.bfloat16


def banner(*a):
    print("CASE", *a, flush=True)


def ints(g, *shape, lo=-3, hi=4, dtype=BF):
    return torch.randint(lo, hi, shape, generator=g, device=DEV).to(dtype)


def normal(g, *shape, dtype=BF, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rounding(dtype):
    return 2.0 ** -8 if dtype == BF else U


def own_error(z, act):
    a = z.abs()
    return {"none": 0 * a, "relu": 0 * a, "silu": (8 + 2 * a) * U * a, "gelu": (16 + a * a) * U * a}[act]


def act64(z, act):
    a, s = O.act(z.double().cpu().numpy(), act)
    return torch.from_numpy(np.asarray(a)).to(DEV), torch.from_numpy(np.asarray(s)).to(DEV)


SIZES = [(1, 8, 8), (1, 72, 56), (2, 136, 1000), (17, 128, 64), (63, 264, 72), (64, 64, 64), (65, 8, 512), (127, 136, 136),
         (129, 1336, 1000), (300, 256, 4096), (16, 1024, 2048), (33, 520, 24), (257, 264, 192), (1000, 768, 256), (5, 2048, 8),
         (777, 1288, 520),
         # few rows: a partial k-step of 64 in either half, more columns than blocks of 8 are for, long reductions
         (8, 72, 24), (7, 64, 104), (9, 64, 104), (3, 5128, 136), (8, 8, 8192), (12, 64, 4104), (4, 5136, 1032),
         # gradients in one launch of large tiles, ragged in all dimensions
         (1001, 1336, 1000), (700, 520, 2056)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_integer_products_are_exact(M, N, K, dtype):
    banner("linear ints", M, N, K, dtype)
    g = gen(M + N + K)
    x, w = ints(g, M, K, dtype=dtype), ints(g, N, K, dtype=dtype)
    b, m, r = ints(g, N, dtype=torch.float32), ints(g, M, N, dtype=dtype), ints(g, M, N, dtype=dtype)
    z = torch.full((M, N), 9.0, device=DEV, dtype=dtype)
    zz = x.double() @ w.double().t() + b.double()
    y = moe.moe_linear(x, w, bias=b, mul=m, residual=r, z=z)
    assert torch.equal(z, zz.to(dtype))
    assert torch.equal(y, (zz * m.double() + r.double()).to(dtype))
    assert torch.equal(moe.moe_linear(x, w), (zz - b.double()).to(dtype))
    assert torch.equal(moe.moe_linear(x, w, act="relu"), (zz - b.double()).clamp(min=0).to(dtype))


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_integer_gradients_are_exact(M, N, K, dtype):
    banner("linear backward ints", M, N, K, dtype)
    g = gen(M + N + K)
    x, w, dy = ints(g, M, K, dtype=dtype), ints(g, N, K, dtype=dtype), ints(g, M, N, dtype=dtype)
    dx, dw, db, dz, dmul = moe.moe_linear_backward(dy, x, w)
    assert dz is dy and dmul is None
    assert torch.equal(dx, (dy.double() @ w.double()).to(dtype))
    full = dy.double().t() @ x.double()
    assert torch.equal(dw, full.float()) and torch.equal(db, dy.double().sum(0).float())
    # a gate without an activation; relu's slope is 0 or 1
    z, m = ints(g, M, N, dtype=dtype), ints(g, M, N, dtype=dtype)
    dx, dw, db, dz, dmul = moe.moe_linear_backward(dy, x, w, z=z, mul=m, act="relu",
                                                   dw_dtype=dtype)
    want = dy.double() * m.double() * (z > 0)
    assert torch.equal(dz, want.to(dtype)) and torch.equal(dmul, (dy.double() * z.double().clamp(min=0)).to(dtype))
    assert torch.equal(db, want.sum(0).float())
    assert torch.equal(dx, (want @ w.double()).to(dtype)) and torch.equal(dw, (want.t() @ x.double()).to(dtype))


# large and ragged in two dimensions, the third one of few chunks: none, one, two, three, with
# and without a partial one
LARGE = [(3601, 3592, n) for n in (40, 64, 72, 128, 200, 320)]


@pytest.mark.parametrize("M,N,K", LARGE + [(M, K, N) for M, N, K in LARGE] + [(K + d, N, M + 7) for d, (M, N, K) in enumerate(LARGE)]
                         # a long reduction in ranges of large tiles; a last round of large tiles cut off the rows
                         + [(9001, 768, 1000), (2422, 14336, 1032), (1032, 2424, 14336), (2422, 1032, 14336)])
def test_large_integer_products_are_exact(M, N, K):
    banner("linear large ints", M, N, K)
    g = gen(M + N + K)
    x, w, dy, r = ints(g, M, K), ints(g, N, K), ints(g, M, N), ints(g, M, N)
    y = moe.moe_linear(x, w, residual=r)
    assert torch.equal(y, (x.double() @ w.double().t() + r.double()).to(BF))
    dx, dw, db, _, _ = moe.moe_linear_backward(dy, x, w)
    assert torch.equal(dx, (dy.double() @ w.double()).to(BF))
    assert torch.equal(dw, (dy.double().t() @ x.double()).float()) and torch.equal(db, dy.double().sum(0).float())


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("M,N,K", [(1, 256, 2048), (65, 264, 1000), (300, 136, 520)])
def test_epilogues(M, N, K, act, dtype):
    banner("linear epilogue", M, N, K, act, dtype)
    g = gen(K)
    x, w = normal(g, M, K, dtype=dtype), normal(g, N, K, dtype=dtype, scale=2 / K ** 0.5)
    b, m, r = normal(g, N, dtype=torch.float32), normal(g, M, N, dtype=dtype), normal(g, M, N, dtype=dtype)
    h = rounding(dtype)
    for bias in (None, b):
        z64 = x.double() @ w.double().t() + (0 if bias is None else bias.double())
        size = x.double().abs() @ w.double().abs().t() + (0 if bias is None else bias.double().abs())
        dz = (K + 2) * U * size
        a = act64(z64, act)[0]
        for mul, res in ((None, None), (m, None), (None, r), (m, r)):
            z = torch.empty((M, N), dtype=dtype, device=DEV)
            y = moe.moe_linear(x, w, bias=bias, act=act, mul=mul, residual=res, z=z)
            assert ((z.double() - z64).abs() <= dz + h * z64.abs()).all()
            want = a if mul is None else a * mul.double()
            tol = 1.13 * dz + own_error(z64, act) + 1e-37
            if mul is not None:
                tol = tol * mul.double().abs() + U * want.abs()
            if res is not None:
                want = want + res.double()
                tol = tol + U * want.abs()
            tol = tol + h * (want.abs() + tol)
            err = (y.double() - want).abs()
            assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "none"])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("M,N,K", [(1, 256, 64), (65, 264, 1000), (900, 136, 72), (1500, 264, 64),
                                   (300, 4232, 64), (1100, 6000, 64)])  # wider than blocks of 32 columns are for
def test_gradients(M, N, K, act, dtype):
    banner("linear backward", M, N, K, act, dtype)
    g = gen(K + 1)
    x, w = normal(g, M, K, dtype=dtype), normal(g, N, K, dtype=dtype, scale=1 / K ** 0.5)
    dy, m = normal(g, M, N, dtype=dtype), normal(g, M, N, dtype=dtype)
    z = normal(g, M, N, dtype=dtype, scale=3.0)
    h = rounding(dtype)
    a, slope = act64(z, act)
    zd = z.double()
    for mul in (None, m):
        if act == "none" and mul is None:
            continue
        dx, dw, db, dz, dmul = moe.moe_linear_backward(dy, x, w, z=z, act=act, mul=mul, dw_dtype=dtype)
        want = dy.double() * slope * (1 if mul is None else mul.double())
        tol = dy.double().abs() * (1 if mul is None else mul.double().abs()) * (own_error(zd, act) / zd.abs().clamp(min=1e-3)
                                                                               * (1 + zd.abs()) + 8 * U)
        tol = tol + 2 * U * want.abs() + 1e-37
        err = (dz.double() - want).abs()
        assert (err <= tol + h * (want.abs() + tol)).all(), float((err / (tol + h * want.abs())).max())
        assert ((db.double() - want.sum(0)).abs() <= tol.sum(0) + (M + 2) * U * want.abs().sum(0)).all()
        if mul is not None:
            wm = dy.double() * a
            tm = dy.double().abs() * own_error(zd, act) + U * wm.abs() + 1e-37
            assert ((dmul.double() - wm).abs() <= tm + h * (wm.abs() + tm)).all()
        else:
            assert dmul is None
        d = dz.double()
        wx, sx = d @ w.double(), d.abs() @ w.double().abs()
        assert ((dx.double() - wx).abs() <= (N + 2) * U * sx + h * (wx.abs() + (N + 2) * U * sx) + 1e-37).all()
        ww, sw = d.t() @ x.double(), d.abs().t() @ x.double().abs()
        assert ((dw.double() - ww).abs() <= (M + 2) * U * sw + h * (ww.abs() + (M + 2) * U * sw) + 1e-37).all()


def test_gradient_against_differences():
    banner("linear differences")
    g = gen(9)
    M, N, K = 5, 16, 24
    x, w, b = (normal(g, *s, dtype=torch.float32) for s in ((M, K), (N, K), (N,)))
    m, r, dy = (normal(g, M, N, dtype=torch.float32) for _ in range(3))
    z = torch.empty((M, N), device=DEV)
    moe.moe_linear(x, w, bias=b, act="gelu", mul=m, residual=r, z=z)
    dx, dw, db, _, dmul = moe.moe_linear_backward(dy, x, w, z=z, act="gelu", mul=m)

    def loss(xx, ww, bb, mm):
        y, _ = O.linear(xx, ww, bb, "gelu", mm, r.double().cpu().numpy())
        return (y * dy.double().cpu().numpy()).sum()

    at = [t.double().cpu().numpy() for t in (x, w, b, m)]
    for n, got in enumerate((dx, dw, db, dmul)):
        got = got.double().cpu().numpy()
        for i in np.random.default_rng(n).integers(0, got.size, 12):
            e = np.zeros(got.size)
            e[i] = 1e-5
            e = e.reshape(got.shape)
            d = (loss(*[v + e if q == n else v for q, v in enumerate(at)]) - loss(*[v - e if q == n else v for q, v in enumerate(at)])) / 2e-5
            # third derivatives' h^2 and fp64's cancellation, and fp32's sums of up to 24 terms
            assert abs(d - got.flat[i]) <= 1e-4 * (1 + abs(d))


def test_padded_weights_and_aliases():
    banner("linear padded")
    g = gen(3)
    M, N, K = 70, 136, 200
    x, w, r = ints(g, M, K), ints(g, N, K), ints(g, M, N)
    wide = torch.full((N, K + 56), float("nan"), device=DEV, dtype=BF)
    wide[:, :K] = w
    want = moe.moe_linear(x, w, residual=r)
    assert torch.equal(moe.moe_linear(x, wide[:, :K], residual=r), want)
    dy = ints(g, M, N)
    assert torch.equal(moe.moe_linear_backward(dy, x, wide[:, :K])[0], moe.moe_linear_backward(dy, x, w)[0])
    y = r.clone()
    assert moe.moe_linear(x, w, residual=y, out=y) is y and torch.equal(y, want)
    want = moe.moe_linear(x, w, mul=r)
    y = r.clone()
    assert torch.equal(moe.moe_linear(x, w, mul=y, out=y), want)
    z = normal(g, M, N)
    ref = moe.moe_linear_backward(dy, x, w, z=z, act="silu")
    d = dy.clone()
    got = moe.moe_linear_backward(d, x, w, z=z, act="silu", dz=d)
    assert all(torch.equal(a, b) for a, b in zip(ref[:4], got[:4]))
    parts = moe.moe_linear_backward(dy, x, w, need_dx=False, need_dbias=False)
    assert parts[0] is None and parts[2] is None and torch.equal(parts[1], moe.moe_linear_backward(dy, x, w)[1])
    assert moe.moe_linear_backward(dy, x, w, need_dw=False)[1] is None


@pytest.mark.parametrize("M,N,K", [(1, 264, 2048), (70, 136, 200), (300, 264, 1000)])
def test_writes_only_its_outputs(M, N, K):
    banner("linear guards", M, N, K)
    g = gen(4)

    def guarded(n, dtype):
        t = torch.full((n + 256,), 7.0, device=DEV, dtype=dtype)
        return t, t[128:128 + n]

    x, w, dy, z, m = ints(g, M, K), ints(g, N, K), ints(g, M, N), ints(g, M, N), ints(g, M, N)
    bufs = [guarded(n, dt) for n, dt in ((M * N, BF), (M * N, BF), (M * K, BF), (N * K, torch.float32), (N, torch.float32),
                                         (M * N, BF), (M * N, BF))]
    v = [b[1] for b in bufs]
    moe.moe_linear(x, w, z=v[0].view(M, N), out=v[1].view(M, N))
    moe.moe_linear_backward(dy, x, w, z=z, mul=m, act="relu", dx=v[2].view(M, K), dw=v[3].view(N, K), dbias=v[4],
                            dz=v[5].view(M, N), dmul=v[6].view(M, N))
    for t, inner in bufs:
        assert (t[:128] == 7).all() and (t[128 + inner.numel():] == 7).all()
    ws = torch.full((moe.linear_ws_bytes(M, N, K, BF) + 512,), 5, dtype=torch.uint8, device=DEV)
    n = ws.numel() - 512
    y = moe.moe_linear(x, w, ws=ws[256:256 + n])
    assert (ws[:256] == 5).all() and (ws[256 + n:] == 5).all() and torch.equal(y, v[1].view(M, N))


def test_no_rows():
    banner("linear M = 0")
    x, w = torch.empty((0, 64), dtype=BF, device=DEV), torch.ones((24, 64), dtype=BF, device=DEV)
    assert moe.moe_linear(x, w).shape == (0, 24)
    dw, db = torch.ones((24, 64), device=DEV), torch.ones(24, device=DEV)
    dx, dw, db, _, _ = moe.moe_linear_backward(torch.empty((0, 24), dtype=BF, device=DEV), x, w, dw=dw, dbias=db)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()


def test_not_finite_rows_stay_in_their_row():
    """A NaN or an infinity in a row of x, or in a tile's neighbour, reaches its row alone."""
    banner("linear NaN rows")
    g = gen(6)
    M, N, K = 130, 136, 72
    x, w = ints(g, M, K), ints(g, N, K)
    want = moe.moe_linear(x, w)
    x2 = x.clone()
    x2[3, 5], x2[64, 71], x2[129, 0] = float("nan"), float("inf"), float("-inf")
    y = moe.moe_linear(x2, w)
    rows = [i for i in range(M) if i not in (3, 64, 129)]
    assert torch.equal(y[rows], want[rows]) and torch.isnan(y[3]).all()
    # columns past a tile's end: a weight row of NaN reaches its column alone
    w2 = w.clone()
    w2[135], w2[64] = float("nan"), float("nan")
    y = moe.moe_linear(x, w2)
    cols = [i for i in range(N) if i not in (64, 135)]
    assert torch.equal(y[:, cols], want[:, cols]) and torch.isnan(y[:, 135]).all()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_graph_and_repeats(M):
    """Captured calls, replayed with other inputs, give the eager calls' bits; calls repeat their own."""
    banner("linear graph", M)
    g = gen(7)
    N, K = 264, 1000
    x, w, dy, z = normal(g, M, K), normal(g, N, K), normal(g, M, N), normal(g, M, N)
    ws = torch.empty(moe.linear_ws_bytes(M, N, K, BF), dtype=torch.uint8, device=DEV)
    wb = torch.empty(moe.linear_backward_ws_bytes(M, N, K, BF), dtype=torch.uint8, device=DEV)
    y = torch.empty((M, N), dtype=BF, device=DEV)
    out = dict(dx=torch.empty_like(x), dw=torch.empty((N, K), device=DEV), dbias=torch.empty(N, device=DEV), dz=torch.empty_like(dy))

    def step():
        moe.moe_linear(x, w, act="silu", residual=z, out=y, ws=ws)
        moe.moe_linear_backward(dy, x, w, z=z, act="silu", ws=wb, **out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.copy_(normal(g, M, K))
        dy.copy_(normal(g, M, N))
        step()
        want = [y.clone()] + [t.clone() for t in out.values()]
        for t in [y] + list(out.values()):
            t.fill_(3.0)
        wb.fill_(255), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [y] + list(out.values())))
