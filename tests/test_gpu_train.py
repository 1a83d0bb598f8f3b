"""GPU tests of the router's training step against float64 (oracle.train_oracle).

Tolerances (fixed before any GPU run), u = 2^-24:
* p: exp to 2 ulp and z - max rounded once, |z - max| <= R: relative 2 (R + 8) u
  =: ep (with the division and the sum of E <= 256 terms in a tree of depth 10).
* losses: sums of terms of one sign, at most 64 fp32 additions a lane before the
  joins: relative ep + 128 u; lse to 2 u (|max| + 10) absolute, which enters lse^2
  times 2 |lse|.
* dlogits: products of p (ep), of c - s (s: ep + 16 u of itself) and of lse, so
  (2 ep + 64 u) of the sizes that the oracle gives, and 2 u (|max| + 10) |g_z| 2 / n p
  of lse's own error.
* dweights and sums along H, T or E of n products: n u sum |a b|.
* rounding to bf16: 2^-8 of the value (half an ulp, 2^-9, on both sides of a
  boundary). Router products in bf16 drop at most 2^-17 of |dz|.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import train_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


def up(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def down(t):
    return t.double().cpu().numpy()


def make(seed, T, E, k, seq, masked, scale=2.0):
    r = np.random.default_rng(seed)
    z = (scale * r.standard_normal((T, E))).astype(np.float32)
    ids = np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)
    mask = None
    if masked:
        mask = (r.random(T) < 0.6).astype(np.uint8) * r.integers(1, 255, T).astype(np.uint8)
        if seq and T > seq:
            mask[:seq] = 0  # a group without live tokens
    v = np.take_along_axis(z.astype(np.float64), ids.astype(np.int64), 1)
    w = np.exp(v - v.max(1, keepdims=True)) if T else v
    w = (w / w.sum(1, keepdims=True) if T else v).astype(np.float32)
    return r, z, ids, mask, w, r.standard_normal((T, k)).astype(np.float32)


def check_balance(z, ids, mask, seq, w, dw, dloss, ws=None):
    """Both kernels on one case; returns the workspace and the outputs."""
    T, E = z.shape
    zz = z if mask is None else np.where((mask != 0)[:, None], z, 0.0)
    fin = zz[np.isfinite(zz).all(1)] if T else zz
    rng = float((fin.max(1) - fin.min(1)).max()) if fin.size else 0.0
    top = float(np.abs(fin).max()) if fin.size else 0.0
    ep = 2 * (min(rng, 104.0) + 8) * U  # exp of less than -104 is 0 in fp32
    loss, counts, live = R.balance(z, ids, mask, seq)
    dm = None if mask is None else up(mask, torch.uint8)
    gl, gc, gv, ws = moe.moe_balance_loss(up(z), up(ids, torch.int32), mask=dm, seq_len=seq, ws=ws)
    assert np.array_equal(gc.cpu().numpy(), counts) and np.array_equal(gv.cpu().numpy(), live)
    assert not ws[:256].any(), "the workspace's ticket is left zero"
    got = down(gl)
    _, lse = R.softmax_rows(zz) if T else (None, np.zeros(1))
    assert abs(got[0] - loss[0]) <= (ep + 128 * U) * loss[0]
    assert abs(got[1] - loss[1]) <= 128 * U * loss[1] + 2 * np.abs(lse).max() * 2 * U * (top + 10)
    outs = []
    for a, b in ((None, None), (w, dw)):
        want, size = R.gate_gradient(z, ids, counts, live, dloss, a, b, mask, seq)
        d = moe.moe_gate_backward(up(z), up(ids, torch.int32), gc, gv, up(np.array(dloss, np.float32)),
                                  weights=None if a is None else up(a), dweights=None if a is None else up(b), mask=dm,
                                  seq_len=seq)
        n = max(1, int(live[-2]))
        tol = (2 * ep + 64 * U) * size + 2 * U * (top + 10) * abs(dloss[1]) * 2.0 / n + 1e-37
        err = np.abs(down(d) - want)
        assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:3])
        outs.append(d)
    return ws, gl, gc, outs


CASES = [
    # T, E, k, seq, masked
    (1, 1, 1, 0, False), (1, 8, 2, 0, False), (64, 8, 2, 0, False), (1000, 8, 2, 0, True), (5, 2, 2, 1, False),
    (33, 3, 1, 11, True), (70, 5, 5, 0, True), (257, 16, 16, 0, False), (96, 60, 4, 32, True), (500, 96, 6, 100, True),
    (31, 128, 8, 0, False), (2048, 128, 1, 512, True), (129, 255, 8, 43, True), (3, 256, 8, 0, False),
    (4096, 256, 8, 1024, True), (5000, 256, 16, 0, True), (600, 253, 16, 1, True),
]


@pytest.mark.parametrize("T,E,k,seq,masked", CASES)
def test_balance(T, E, k, seq, masked):
    banner("balance", T, E, k, seq, masked)
    r, z, ids, mask, w, dw = make(T + E, T, E, k, seq, masked)
    check_balance(z, ids, mask, seq, w, dw / T, (0.7, -0.3))


def test_balance_shared_workspace_and_repeats():
    """One workspace through calls of other sizes; a repeated call is the same bits."""
    banner("balance workspace")
    ws = torch.zeros(moe.balance_ws_bytes(4096, 256, 8, 1024) * 2, dtype=torch.uint8, device=DEV)
    first = None
    for T, E, k, seq in ((4096, 256, 8, 1024), (64, 8, 2, 0), (600, 60, 4, 1), (4096, 256, 8, 1024)):
        _, z, ids, mask, w, dw = make(7, T, E, k, seq, True)
        ws, gl, gc, outs = check_balance(z, ids, mask, seq, w, dw, (1.0, 0.1), ws=ws)
        if T == 4096 and first is not None:
            assert torch.equal(gl, first[0]) and all(torch.equal(a, b) for a, b in zip(outs, first[1]))
        if T == 4096:
            first = (gl, outs)


def test_balance_masked_values_and_odd_ids():
    """Masked rows may hold anything; ids outside [0, E) are not counted and get no
    gradient; rows of -inf and single -inf logits (masked experts) are defined."""
    banner("balance odd values")
    _, z, ids, mask, w, dw = make(21, 80, 60, 4, 20, True)
    dead = np.flatnonzero(mask == 0)
    z[dead[0]], z[dead[1]], z[dead[2]] = np.nan, np.inf, -np.inf
    live = np.flatnonzero(mask)
    z[live[0]] = -np.inf
    z[live[1], 5:] = -np.inf
    z[live[2], ::2] = np.finfo(np.float32).min
    ids[live[3], 1], ids[live[4], 0] = -1, 60
    ids[live[5], 2] = 2 ** 30
    check_balance(z, ids, mask, 20, w, dw, (1.0, 0.5))


def test_balance_nan_and_inf_show():
    banner("balance nan")
    for bad in (np.nan, np.inf):
        _, z, ids, _, w, dw = make(22, 40, 16, 2, 0, False)
        z[7, 3] = bad
        l, c, v, _ = moe.moe_balance_loss(up(z), up(ids, torch.int32))
        assert torch.isnan(l[0])
        d = moe.moe_gate_backward(up(z), up(ids, torch.int32), c, v, torch.ones(2, device=DEV))
        assert torch.isnan(d[7, 3]) and torch.isfinite(d[:7]).all() and torch.isfinite(d[8:]).all()


def test_balance_all_masked_and_empty():
    banner("balance empty")
    _, z, ids, _, w, dw = make(23, 24, 8, 2, 6, False)
    check_balance(z, ids, np.zeros(24, np.uint8), 6, w, dw, (1.0, 1.0))
    for seq, G in ((0, 1), (5, 0)):
        l, c, v, _ = moe.moe_balance_loss(torch.empty((0, 8), device=DEV), torch.empty((0, 2), dtype=torch.int32, device=DEV),
                                          seq_len=seq)
        assert l.tolist() == [0, 0] and tuple(c.shape) == (G, 8) and not c.any() and v.tolist() == [0] * (G + 2)


def test_balance_large_logits():
    banner("balance large logits")
    _, z, ids, _, w, dw = make(24, 200, 32, 4, 0, False, scale=60.0)
    check_balance(z, ids, None, 0, w, dw, (1.0, 0.01))


def test_gate_gradient_against_differences():
    """The kernel's gradient along a direction against the float64 losses' difference."""
    banner("gate differences")
    r, z, ids, mask, _, _ = make(25, 96, 24, 3, 32, True)
    g = np.array([0.9, 0.2])
    loss, counts, live = R.balance(z, ids, mask, 32)
    _, c, v, _ = moe.moe_balance_loss(up(z), up(ids, torch.int32), mask=up(mask, torch.uint8), seq_len=32)
    d = down(moe.moe_gate_backward(up(z), up(ids, torch.int32), c, v, up(g), mask=up(mask, torch.uint8), seq_len=32))
    for _ in range(8):
        a = r.standard_normal(z.shape)
        h = 1e-4
        num = (R.balance(z + h * a, ids, mask, 32)[0] - R.balance(z - h * a, ids, mask, 32)[0]) @ g / (2 * h)
        assert abs(num - (d * a).sum()) <= 1e-5 * np.abs(d * a).sum()


# ---------------------------------------------------------------- combine
@pytest.mark.parametrize("T,k,H,dtype", [(1, 1, 8, torch.bfloat16), (1, 8, 7168, torch.bfloat16), (5, 2, 4, torch.float32),
                                         (64, 2, 128, torch.float32), (37, 16, 520, torch.bfloat16),
                                         (130, 8, 2048, torch.bfloat16), (33, 3, 1036, torch.float32)])
def test_combine_backward(T, k, H, dtype):
    banner("combine", T, k, H, dtype)
    r = np.random.default_rng(T + H)
    n = T * k
    M = n + 3
    local = r.random(n) < 0.6
    if T > 2:
        local[:k] = False  # a token without local experts
    dest = np.full(n, -1, np.int32)
    dest[local] = r.permutation(M)[: local.sum()]
    if T > 4:
        dest[k], dest[k + 1] = M, -7  # outside the rows: as remote
    do, y = up(r.standard_normal((T, H)), dtype), up(r.standard_normal((M, H)), dtype)
    w = r.random((T, k)).astype(np.float32)
    dy = torch.full((M, H), 9.0, dtype=dtype, device=DEV)
    dw, got = moe.moe_combine_backward(do, y, up(w), up(dest, torch.int32), dy_perm=dy)
    want, size, rows = R.combine_gradient(down(do), down(y), w, dest)
    assert (np.abs(down(dw) - want) <= H * U * size).all()
    f = down(dy)
    for row in range(M):
        if row in rows:
            t, j = rows[row]
            exact = w[t, j].astype(np.float64) * down(do[t])
            assert (np.abs(f[row] - exact) <= (2.0 ** -8 if dtype == torch.bfloat16 else U) * np.abs(exact)).all()
        else:
            assert (f[row] == 9.0).all()
    dw2, none = moe.moe_combine_backward(do, y, up(w), up(dest, torch.int32), need_dy=False)
    assert none is None and torch.equal(dw2, dw)


def test_combine_backward_undoes_the_layer():
    """On the layer's own dispatch: <dout, combine(y, w)> is linear in w, and dw its gradient."""
    banner("combine layer")
    T, k, E, H = 200, 4, 16, 256
    r = np.random.default_rng(5)
    ids = up(np.stack([r.permutation(E)[:k] for _ in range(T)]), torch.int32)
    emap = np.where(np.arange(E) % 2 == 0, np.arange(E) // 2, -1).astype(np.int32)
    _, off, ws = moe.moe_expert_histogram_scan(ids, E, emap)
    x = torch.randn((T, H), device=DEV)
    _, _, dest = moe.moe_permute(x, ids, emap, ws, gather=False)
    y, w, do = torch.randn((T * k, H), device=DEV), torch.rand((T, k), device=DEV), torch.randn((T, H), device=DEV)
    dw, _ = moe.moe_combine_backward(do, y, w, dest)
    out = moe.moe_unpermute_combine(y, w, dest, T)
    a, b = (do.double() * out.double()).sum(1), (dw.double() * w.double()).sum(1)
    size = (do.abs().double() * out.abs().double()).sum(1) + 1e-3
    assert ((a - b).abs() <= 1e-4 * size).all()


# ---------------------------------------------------------------- router product
ROUTER = [
    (0, 8, 64), (1, 1, 64), (1, 256, 7168), (3, 5, 128), (31, 8, 192), (32, 60, 64), (33, 64, 320), (65, 96, 2048),
    (129, 128, 1024), (500, 200, 448), (700, 255, 128), (1000, 256, 2048), (4099, 128, 512), (2049, 256, 5120),
]


@pytest.mark.parametrize("T,E,H", ROUTER)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_router_grad(T, E, H, dtype):
    banner("router", T, E, H, dtype)
    r = np.random.default_rng(T + E + H)
    dz = torch.from_numpy(r.standard_normal((T, E)) * np.exp(r.standard_normal((T, 1)))).float().to(DEV)
    x, w = up(r.standard_normal((T, H)), dtype), up(r.standard_normal((E, H)) / np.sqrt(H), dtype)
    dx, dw, db, ws = moe.moe_router_grad(dz, x, w)
    a, b, c = dz.double(), x.double(), w.double()
    cut = 2.0 ** -17 if dtype == torch.bfloat16 else 0.0
    want, size = a.t() @ b, a.abs().t() @ b.abs()
    assert ((dw.double() - want).abs() <= (cut + (2 * T + 8) * U) * size).all()
    want, size = a.sum(0), a.abs().sum(0)
    assert ((db.double() - want).abs() <= (T + 8) * U * size).all()
    want, size = a @ c, a.abs() @ c.abs()
    tol = (cut + 2 * E * U) * size + (2.0 ** -8 * want.abs() if cut else 0.0)
    assert ((dx.double() - want).abs() <= tol).all()
    none, dw2, db2, _ = moe.moe_router_grad(dz, x, w, ws=ws, need_dx=False)
    assert none is None and torch.equal(dw2, dw) and torch.equal(db2, db), "a repeated call differs"


def test_router_grad_outputs_stay_in_bounds():
    """Rows past T and past E of larger buffers are left alone."""
    banner("router bounds")
    T, E, H = 45, 37, 192
    dz, x = torch.randn((T, E), device=DEV), torch.randn((T, H), device=DEV).bfloat16()
    w = torch.randn((E, H), device=DEV).bfloat16()
    dx = torch.full((T + 200, H), 3.0, dtype=torch.bfloat16, device=DEV)
    dw = torch.full((E + 300, H), 3.0, device=DEV)
    db = torch.full((E + 300,), 3.0, device=DEV)
    moe.moe_router_grad(dz, x, w, dx=dx[:T], dw=dw[:E], dbias=db[:E])
    assert (dx[T:] == 3.0).all() and (dw[E:] == 3.0).all() and (db[E:] == 3.0).all()


def test_router_grad_nan_stays_in_its_row_and_column():
    banner("router nan")
    T, E, H = 100, 40, 256
    dz, x = torch.randn((T, E), device=DEV), torch.randn((T, H), device=DEV).bfloat16()
    w = torch.randn((E, H), device=DEV).bfloat16()
    dz[99, 7] = float("nan")
    x[98, 9] = float("inf")
    dx, dw, db, _ = moe.moe_router_grad(dz, x, w)
    assert torch.isnan(dx[99]).all() and torch.isfinite(dx[:99]).all()
    assert torch.isnan(dw[7]).all() and torch.isnan(db[7]) and torch.isfinite(db[:7]).all()
    ok = torch.ones(H, dtype=torch.bool, device=DEV)
    ok[9] = False
    assert torch.isfinite(dw[:7][:, ok]).all() and not torch.isfinite(dw[:, 9]).any()


# ---------------------------------------------------------------- streams, graphs, refusals
def test_training_step_on_another_stream_and_in_a_graph():
    banner("train graph")
    T, E, k, H = 300, 32, 4, 256
    cases = [make(s, T, E, k, 100, True) for s in (1, 2, 3)]
    x, rw = torch.randn((T, H), device=DEV).bfloat16(), torch.randn((E, H), device=DEV).bfloat16()
    g = torch.tensor([0.3, 0.1], device=DEV)
    ws = torch.zeros(moe.balance_ws_bytes(T, E, k, 100), dtype=torch.uint8, device=DEV)
    rws = torch.empty(moe.router_grad_ws_bytes(T, E, H, x.dtype), dtype=torch.uint8, device=DEV)

    def step(z, ids, mask, w, dw):
        loss, counts, live, _ = moe.moe_balance_loss(z, ids, mask=mask, seq_len=100, ws=ws)
        dz = moe.moe_gate_backward(z, ids, counts, live, g, weights=w, dweights=dw, mask=mask, seq_len=100)
        dx, dwr, db, _ = moe.moe_router_grad(dz, x, rw, ws=rws)
        return [loss, counts, dz, dx, dwr, db]

    ins = [[up(z), up(i, torch.int32), up(m, torch.uint8), up(w), up(d)] for _, z, i, m, w, d in cases]
    want = [step(*i) for i in ins]
    buf = [t.clone() for t in ins[0]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(*buf)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*buf)
    for i in (1, 2, 0, 1):
        for b, t in zip(buf, ins[i]):
            b.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), i


def test_refusals():
    banner("train refusals")
    z, ids = torch.randn((6, 8), device=DEV), torch.zeros((6, 2), dtype=torch.int32, device=DEV)
    l, c, v, ws = moe.moe_balance_loss(z, ids)
    one = torch.ones(2, device=DEV)
    for bad in (lambda: moe.moe_balance_loss(z.double(), ids), lambda: moe.moe_balance_loss(z, ids[:5]),
                lambda: moe.moe_balance_loss(z, ids, seq_len=4), lambda: moe.moe_balance_loss(z, ids, seq_len=-1),
                lambda: moe.moe_balance_loss(z, ids, mask=torch.ones(5, dtype=torch.uint8, device=DEV)),
                lambda: moe.moe_balance_loss(z, ids.long()), lambda: moe.moe_balance_loss(z.t(), ids),
                lambda: moe.moe_balance_loss(z.cpu(), ids), lambda: moe.moe_balance_loss(z, ids, counts=c[:, :4]),
                lambda: moe.moe_gate_backward(z, ids, c, v, one, weights=torch.ones((6, 2), device=DEV)),
                lambda: moe.moe_gate_backward(z, ids, c[:, :7], v, one), lambda: moe.moe_gate_backward(z, ids, c, v, one[:1]),
                lambda: moe.moe_combine_backward(z, z, torch.ones((6, 2), device=DEV), torch.zeros(11, dtype=torch.int32, device=DEV)),
                lambda: moe.moe_router_grad(z, torch.randn((6, 64), device=DEV), torch.randn((8, 64), device=DEV).bfloat16()),
                lambda: moe.moe_router_grad(z, torch.randn((6, 64), device=DEV), torch.randn((7, 64), device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(moe.MoeError):
        moe.moe_balance_loss(z, torch.zeros((6, 9), dtype=torch.int32, device=DEV))
    with pytest.raises(moe.MoeError):
        moe.moe_router_grad(z, torch.randn((6, 96), device=DEV).bfloat16(), torch.randn((8, 96), device=DEV).bfloat16())
    with pytest.raises(moe.MoeError):
        moe.moe_combine_backward(torch.randn((6, 6), device=DEV), torch.randn((12, 6), device=DEV),
                                 torch.ones((6, 2), device=DEV), torch.zeros(12, dtype=torch.int32, device=DEV))
