"""CPU oracle of the router's training step, in float64. TEST INFRASTRUCTURE ONLY
(see ``moe_oracle``). Shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def softmax_rows(z):
    """p and lse of rows; a row of -inf alone has p = 0 and lse = 0."""
    z = np.asarray(z, np.float64)
    m = z.max(1, keepdims=True)
    none = np.isneginf(m)
    e = np.exp(z - np.where(none, 0.0, m))
    s = e.sum(1, keepdims=True)
    p = np.where(none, 0.0, e / np.where(none, 1.0, s))
    lse = np.where(none, 0.0, np.where(none, 0.0, m) + np.log(np.where(none, 1.0, s)))
    return p, lse[:, 0]


def _groups(T, seq):
    return [np.arange(T)] if not seq else [np.arange(a, a + seq) for a in range(0, T, seq)]


def balance(z, ids, mask=None, seq=0):
    """(losses [2], counts [groups, E], live [groups + 2])."""
    T, E = z.shape
    k = ids.shape[1]
    on = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    z = np.where(on[:, None], z, 0.0)
    p, lse = softmax_rows(z) if T else (np.zeros((0, E)), np.zeros(0))
    groups = _groups(T, seq)
    counts = np.zeros((len(groups), E), np.int64)
    live, terms = [], []
    for g, rows in enumerate(groups):
        rows = rows[on[rows]]
        i = ids[rows].ravel()
        counts[g] = np.bincount(i[(i >= 0) & (i < E)], minlength=E)
        live.append(len(rows))
        if len(rows):
            terms.append((counts[g] * E / (k * len(rows)) * p[rows].mean(0)).sum())
    n = sum(live)
    losses = np.array([np.mean(terms) if terms else 0.0, (lse[on] ** 2).sum() / n if n else 0.0])
    return losses, counts, np.array(live + [n, len(terms)])


def gate_gradient(z, ids, counts, live, dloss, w=None, dw=None, mask=None, seq=0):
    """(dlogits, bound): the gradient and, per element, the size of the terms that
    a rounding of p, of the sums and of the products acts on."""
    T, E = z.shape
    k = ids.shape[1]
    on = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    p, lse = softmax_rows(np.where(on[:, None], z, 0.0))
    d, size = np.zeros((T, E)), np.zeros((T, E))
    n, full = int(live[-2]), int(live[-1])
    for g, rows in enumerate(_groups(T, seq)):
        rows = rows[on[rows]]
        if len(rows) == 0:
            continue
        f = float(dloss[0]) / full * E / (k * float(len(rows)) ** 2)
        c = counts[g].astype(np.float64)
        s = p[rows] @ c
        zt = float(dloss[1]) * 2.0 / n * lse[rows]
        d[rows] = p[rows] * (f * (c - s[:, None]) + zt[:, None])
        size[rows] = p[rows] * (abs(f) * (c + s[:, None]) + np.abs(zt)[:, None])
    if w is not None:
        w, dw = np.asarray(w, np.float64), np.asarray(dw, np.float64)
        t = w * (dw - (w * dw).sum(1, keepdims=True))
        u = np.abs(w) * (np.abs(dw) + np.abs(w * dw).sum(1, keepdims=True))
        for j in range(k):
            ok = (ids[:, j] >= 0) & (ids[:, j] < E)
            r = np.arange(T)[ok]
            np.add.at(d, (r, ids[ok, j]), t[ok, j])
            np.add.at(size, (r, ids[ok, j]), u[ok, j])
    return d, size


def combine_gradient(dout, y, w, dest):
    """(dw [T, k], size of dw's terms, {row: (dy row)})."""
    T, k = w.shape
    dest = np.asarray(dest).reshape(T, k)
    dw, size, dy = np.zeros((T, k)), np.zeros((T, k)), {}
    for t in range(T):
        for j in range(k):
            r = int(dest[t, j])
            if 0 <= r < y.shape[0]:
                dw[t, j] = dout[t] @ y[r]
                size[t, j] = np.abs(dout[t]) @ np.abs(y[r])
                dy[r] = (t, j)
    return dw, size, dy
