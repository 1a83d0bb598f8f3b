"""GPU tests of scored, group-limited routing and its gradient against the float64 oracle.

Tolerances (fixed before any GPU run), u = 2^-24:
* ids: equal. Scores that decide are held in 64 bits on both sides;
* weights: fp32. Let d be the largest difference between logits that enter a weight (for a
  sigmoid by itself 0). An exponential is off by its argument's rounding, u d, and its own 2 u; a
  sigmoid by that, a sum and a quotient: (d + 4) u. A ratio of up to 16 of them: twice (d + 6) u,
  4 u for the tree of the sum, 2 u for quotient and scale: (2 d + 18) u. A softmax by itself: its
  sum is off by the mean of its terms' errors, (2.5 d' + 3) u with d' their mean distance from the
  largest (at most log 256, so 17 u), and 20 additions; reciprocal, product and scale 5 u; the
  exponential (d + 2) u: (d + 44) u in all. So (2 d + 48) u of the value, and gradual underflow,
  scaled by at most 2.5: 2^-147;
* gradients: fp32. A sigmoid or exponential of an argument that is exact, or a difference of
  two exact ones (u of an argument of at most 30, hence 30 u of the value), is off by 36 u with
  the function's own 2 ulp (4 u) and the division; the sums over at most 16 slots and 256
  columns (an exponential's sum: its terms' errors and 8 steps of a tree of 64 lanes of 4)
  add 12 u each. The formulas have at most three such factors: 256 u of the sum of the sizes of
  the terms: for a slot |w_j| (|dw_j| + sum_i r_i |dw_i|).
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


def up(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def check_route(z, k, **kw):
    ids, w = moe.moe_route(up(z), k, **{n: up(v, torch.uint8 if n == "mask" else torch.float32) if isinstance(v, np.ndarray) else v
                                        for n, v in kw.items()})
    want_ids, want = O.route(z, k, **kw)
    wrong = np.flatnonzero((ids.cpu().numpy() != want_ids).any(1))
    assert wrong.size == 0, ("ids", wrong[:5], ids[wrong[:1]].tolist(), want_ids[wrong[:1]].tolist())
    got = w.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    d = np.zeros((len(z), 1))
    for t in range(len(z)):
        sel = z[t][want_ids[t][want_ids[t] >= 0]].astype(np.float64)
        fin = sel[np.isfinite(sel)]
        if fin.size and (kw.get("norm", True) or kw.get("score") == "softmax"):
            d[t] = (fin.max() if kw.get("norm", True) else z[t][np.isfinite(z[t])].max()) - fin.min()
    tol = (2 * d + 48) * U * np.abs(want) + 2.0 ** -147
    ratio = float((np.abs(got - want) / tol)[ok].max())
    assert ratio <= 1.0
    return ids, w


CONFIGS = [(8, 2, 1, 1), (1, 1, 1, 1), (60, 4, 1, 1), (60, 4, 5, 2), (64, 16, 4, 2), (65, 3, 13, 4), (128, 8, 8, 3),
           (160, 6, 8, 3), (192, 9, 3, 2), (256, 8, 8, 4), (256, 16, 1, 1), (256, 8, 256, 20), (256, 16, 128, 8),
           (250, 7, 2, 1), (100, 10, 100, 100)]


@pytest.mark.parametrize("E,k,G,g", CONFIGS)
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_route(E, k, G, g, score):
    banner("route", E, k, G, g, score)
    r = np.random.default_rng(E * 100 + k)
    for T in (1, 3, 65, 258):
        z = (2 * r.standard_normal((T, E))).astype(np.float32)
        b = (0.2 * r.standard_normal(E)).astype(np.float32)
        check_route(z, k, score=score, bias=b if T != 3 else None, n_group=G, topk_group=g, norm=T % 2 == 1, scale=2.5,
                    mask=(r.random(T) < 0.7).astype(np.uint8) if T > 3 else None)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,k,G,g", [(256, 8, 8, 4), (60, 4, 5, 2), (8, 3, 1, 1)])
def test_route_ties(E, k, G, g, score):
    """Logits on a coarse grid: rows full of equal scores, equal groups too."""
    banner("route ties", E, k, G, g, score)
    r = np.random.default_rng(3)
    z = r.integers(-2, 3, (130, E)).astype(np.float32)
    z[:10] = 0.5
    check_route(z, k, score=score, n_group=G, topk_group=g)
    check_route(z, k, score=score, n_group=G, topk_group=g, bias=(r.integers(0, 2, E) / 4).astype(np.float32))


def test_route_scores_that_fp32_cannot_tell_apart():
    """Biases that bring c's of different scores within 2^-30 of each other."""
    banner("route near ties")
    r = np.random.default_rng(4)
    E = 64
    for T in (40,):
        z = r.standard_normal((T, E)).astype(np.float32)
        # the bias makes c nearly constant for row 0's logits: what is left is its rounding
        b = (1.0 - O.scores(z[0], "sigmoid")).astype(np.float32)
        z[:] = z[0]
        check_route(z, 8, bias=b)
        check_route(z, 8, bias=b, n_group=8, topk_group=3)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("G,g", [(1, 1), (4, 2)])
def test_route_masked_and_bad_logits(score, G, g):
    banner("route bad", score, G, g)
    r = np.random.default_rng(5)
    E, k = 32, 6
    z = r.standard_normal((40, E)).astype(np.float32)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, 7] = 0.25
    z[2, :30] = -np.inf
    z[3, 5] = np.nan
    z[4] = np.nan
    z[5, 3] = np.inf
    z[6, 3:9] = np.inf
    z[7] = np.finfo(np.float32).min
    z[8] = -800.0
    z[9] = np.finfo(np.float32).max
    z[10, ::2] = -np.inf
    z[11, 8:] = -np.inf
    z[12] = -100.0 - np.arange(E)
    z[13, 0], z[13, 1] = 88.0, -88.0
    with np.errstate(over="ignore", invalid="ignore"):
        check_route(z, k, score=score, n_group=G, topk_group=g)
        check_route(z, k, score=score, n_group=G, topk_group=g, norm=False)
        b = np.zeros(E, np.float32)
        b[2], b[9], b[20], b[21] = -np.inf, np.inf, np.nan, -3.0
        check_route(z, k, score=score, n_group=G, topk_group=g, bias=b)
        mask = np.ones(40, np.uint8)
        mask[[3, 4, 5, 20]] = 0  # what masked rows hold does not matter
        mask[30] = 255
        check_route(z, k, score=score, n_group=G, topk_group=g, mask=mask)


def grad_tolerance(z, ids, dw, score, norm, scale):
    T, E = z.shape
    tol = np.full((T, E), 2.0 ** -140)
    for t in range(T):
        s = O.scores(z[t], score)
        at = [(j, e) for j, e in enumerate(ids[t]) if 0 <= e < E]
        r = O.ratios([z[t, e] for _, e in at], score) if norm else s[[e for _, e in at]]
        mean = (r * np.abs([dw[t, j] for j, _ in at])).sum()
        for (j, e), x in zip(at, r):
            tol[t, e] += 256 * U * scale * x * (abs(dw[t, j]) + mean)
        if score == "softmax" and not norm:
            tol[t] += 256 * U * scale * s * mean
    return tol


@pytest.mark.parametrize("E,k", [(1, 1), (8, 2), (60, 4), (64, 16), (65, 3), (160, 6), (256, 8), (250, 16)])
@pytest.mark.parametrize("score,norm", [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)])
def test_route_backward(E, k, score, norm):
    banner("route backward", E, k, score, norm)
    r = np.random.default_rng(E + k)
    for T in (1, 5, 131):
        z = (2 * r.standard_normal((T, E))).astype(np.float32)
        ids = np.argsort(r.random((T, E)), 1)[:, :k].astype(np.int32)
        dw = r.standard_normal((T, k)).astype(np.float32)
        if T > 1:
            z[0] = -np.inf
            z[1, ids[1, 0]] = -np.inf
            z[2] *= 12
            ids[3, 0], ids[4, -1] = -1, E  # slots without an expert
            ids[4, 0] = np.iinfo(np.int32).min
        if T > 100 and k > 1:
            ids[5, 1] = ids[5, 0]  # the same expert twice
            ids[6] = -1
            z[7] = -120.0 - np.arange(E) / 16
            z[8] = 95.0
        dz = moe.moe_route_backward(up(z), up(ids, torch.int32), up(dw), score=score, norm=norm, scale=1.5)
        with np.errstate(invalid="ignore", over="ignore"):
            want = O.route_backward(z, ids, dw, score, norm, 1.5)
            tol = grad_tolerance(z, ids, dw, score, norm, 1.5)
        err = np.abs(dz.cpu().numpy() - want)
        wrong = np.argwhere(~(err <= tol))
        assert wrong.size == 0, (T, float((err / tol).max()), wrong[:5])
        base = torch.randn((T, E), device=DEV)
        acc = moe.moe_route_backward(up(z), up(ids, torch.int32), up(dw), score=score, norm=norm, scale=1.5,
                                     dlogits=base.clone(), accumulate=True)
        assert torch.equal(acc, base + dz)


def test_route_writes_only_its_outputs():
    banner("route guards")
    T, E, k = 37, 60, 4
    z = torch.randn((T, E), device=DEV)
    ids = torch.full((T * k + 64,), 77, dtype=torch.int32, device=DEV)
    w = torch.full((T * k + 64,), 7.0, device=DEV)
    moe.moe_route(z, k, ids=ids[32:32 + T * k].view(T, k), weights=w[32:32 + T * k].view(T, k))
    assert (ids[:32] == 77).all() and (ids[32 + T * k:] == 77).all() and (ids[32:32 + T * k] < E).all()
    assert (w[:32] == 7).all() and (w[32 + T * k:] == 7).all()
    d = torch.full((T * E + 64,), 7.0, device=DEV)
    moe.moe_route_backward(z, ids[32:32 + T * k].view(T, k), torch.randn((T, k), device=DEV), dlogits=d[32:32 + T * E].view(T, E))
    assert (d[:32] == 7).all() and (d[32 + T * E:] == 7).all()


def test_route_ids_through_the_dispatch():
    """Slots without an expert pass through histogram, permutation and combine."""
    banner("route dispatch")
    T, E, k, H = 50, 16, 4, 128
    z = torch.randn((T, E), device=DEV)
    z[3] = float("-inf")
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[40:] = 0
    ids, w = moe.moe_route(z, k, n_group=4, topk_group=2, mask=mask)
    x = torch.randn((T, H), device=DEV).bfloat16()
    emap = np.arange(E, dtype=np.int32)
    counts, offsets, ws = moe.moe_expert_histogram_scan(ids, E, emap)
    x_perm, src, dest = moe.moe_permute(x, ids, emap, ws)
    assert int(counts.sum()) == 39 * k == int(offsets[-1])
    dest = dest.view(T, k)
    assert (dest[40:] == -1).all() and (dest[3] == -1).all() and (dest[:3] >= 0).all()
    out = moe.moe_unpermute_combine(x_perm, w, dest.view(-1), T)
    assert (out[40:] == 0).all() and (out[3] == 0).all()
    assert torch.allclose(out[:3].float(), x[:3].float(), atol=2e-2)  # normalised weights of the row itself
