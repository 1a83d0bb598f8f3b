"""Oracle of what stands around the routed experts: scored, group-limited routing and its
gradient, dense products with an epilogue and their gradients, dropout from a
counter-based generator. numpy, float64, one row at a time where that is plainer.
"""
from __future__ import annotations

import math

import numpy as np


def scores(z, score):
    z = np.asarray(z, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-z))
        if not np.any(z > -np.inf):
            return np.zeros_like(z)
        e = np.exp(z - np.max(z))
        return e / e.sum()


def ratios(z, score):
    """Scores of the logits z over their sum, where the scores underflow too."""
    z = np.asarray(z, np.float64)
    if not z.size or z.max() == -np.inf:
        return np.zeros_like(z)
    logs = -np.logaddexp(0.0, -z) if score == "sigmoid" else z - z.max()
    r = np.exp(logs - logs.max())
    return r / r.sum()


def route(logits, k, score="sigmoid", bias=None, mask=None, n_group=1, topk_group=1, norm=True, scale=1.0):
    """(ids [T, k], weights [T, k]) of moe_route."""
    T, E = logits.shape
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    b = np.zeros(E) if bias is None else np.asarray(bias, np.float64)
    n = E // n_group
    for t in range(T):
        if mask is not None and mask[t] == 0:
            continue
        z = np.asarray(logits[t], np.float64)
        out = np.isnan(z) | (z == np.inf if score == "softmax" else np.zeros(E, bool))
        bad = bool(out.any())
        s = scores(np.where(out, -np.inf, z), score)
        with np.errstate(invalid="ignore"):
            c = s + b
        can = ~out & (z > -np.inf) & (c > -np.inf)
        c = np.where(can, c, -np.inf)
        if topk_group < n_group:
            best = np.empty(n_group)
            for g in range(n_group):
                top = np.sort(c[g * n:(g + 1) * n])[::-1][:2]
                top = top[top > -np.inf]
                best[g] = top.sum() if top.size else -np.inf
            kept = sorted(range(n_group), key=lambda g: (-best[g], g))[:topk_group]
            for g in range(n_group):
                if g not in kept:
                    c[g * n:(g + 1) * n] = -np.inf
        order = [e for e in sorted(range(E), key=lambda e: (-c[e], e)) if c[e] > -np.inf][:k]
        ids[t, :len(order)] = order
        w[t, :len(order)] = scale * (ratios(z[order], score) if norm else s[order])
        if bad:
            w[t] = np.nan
    return ids, w


def route_backward(logits, ids, dw, score="sigmoid", norm=True, scale=1.0):
    """dlogits [T, E]: the weights' Jacobian, step by step."""
    T, E = logits.shape
    dz = np.zeros((T, E))
    for t in range(T):
        z = np.asarray(logits[t], np.float64)
        s = scores(z, score)
        slots = [(j, int(e)) for j, e in enumerate(ids[t]) if 0 <= e < E]
        if not slots:  # no weight depends on these logits, whatever they hold
            continue
        d = scale * np.array([float(dw[t, j]) for j, _ in slots])
        if norm:
            r = ratios([z[e] for _, e in slots], score)
            d = d - (r * d).sum()  # times s / (their sum) = r below
            if score == "softmax":
                for (j, e), x in zip(slots, r * d):
                    dz[t, e] += x
                continue
            with np.errstate(over="ignore"):
                for (j, e), x in zip(slots, r * d):
                    dz[t, e] += x / (1.0 + math.exp(min(z[e], 700.0)))
            continue
        if score == "sigmoid":
            for (j, e), x in zip(slots, d):
                dz[t, e] += x * s[e] / (1.0 + math.exp(min(z[e], 700.0)))
        else:
            ds = np.zeros(E)
            for (j, e), x in zip(slots, d):
                ds[e] += x
            dz[t] = s * (ds - (s * ds).sum())
    return dz


def act(z, name):
    """The activation and its derivative."""
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    with np.errstate(over="ignore"):
        if name == "silu":
            q, r = 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))
            return z * q, q + z * q * r
    if name == "gelu":
        q = 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-z / math.sqrt(2.0))
        return z * q, q + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return z, np.ones_like(z)


def linear(x, w, bias=None, name="none", mul=None, residual=None):
    """(y, z) of moe_linear, not rounded."""
    z = x.astype(np.float64) @ w.astype(np.float64).T
    if bias is not None:
        z = z + bias
    y = act(z, name)[0]
    if mul is not None:
        y = y * mul
    if residual is not None:
        y = y + residual
    return y, z


def act_backward(dy, z=None, name="none", mul=None):
    """(dz, dmul) of moe_linear_backward, not rounded."""
    dy = np.asarray(dy, np.float64)
    a, slope = act(z, name) if z is not None else (None, 1.0)
    dz = dy * slope * (1.0 if mul is None else mul)
    return dz, None if mul is None else dy * a


def philox(counter, key):
    """Four 32-bit words of Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw 2011):
    counter of four words, key of two."""
    c, k = list(counter), list(key)
    for _ in range(10):
        u, v = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(v >> 32) ^ c[1] ^ k[0], v & 0xFFFFFFFF, (u >> 32) ^ c[3] ^ k[1], u & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_words(n, seed, offset):
    """The words of n elements."""
    out = np.empty(4 * ((n + 3) // 4), np.uint64)
    m = (1 << 64) - 1
    for q in range((n + 3) // 4):
        c = (offset + q) & m
        out[4 * q:4 * q + 4] = philox((c & 0xFFFFFFFF, c >> 32, 0, 0), (seed & 0xFFFFFFFF, (seed & m) >> 32))
    return out[:n]


def dropout_add(x, p, seed, offset, residual=None):
    """fp64 values of moe_dropout_add (its factor is fl32(1 / (1 - p)))."""
    keep = dropout_words(x.size, seed, offset).reshape(x.shape) >= math.floor(p * 4294967296.0)
    with np.errstate(invalid="ignore"):
        y = np.where(keep, x.astype(np.float64) * float(np.float32(1.0 / (1.0 - p))), 0.0)
    return y if residual is None else y + residual
