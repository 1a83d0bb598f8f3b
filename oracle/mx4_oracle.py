"""CPU oracle for MXFP4. TEST INFRASTRUCTURE ONLY (see ``mx_oracle``).

OCP Microscaling FP4: E2M1 elements (sign, 2 exponent bits, 1 mantissa bit: 0,
0.5, 1, 1.5, 2, 3, 4, 6) sharing one E8M0 scale 2^(c - 127) per 32 consecutive
elements. Quantising a block: shared exponent floor(log2(max |v|)) - 2 (2 is the
exponent of E2M1's largest power of two), clamped to at least -127 (an all-zero
block takes it); element = RNE_E2M1(clamp(v / 2^s, -6, 6)), ties to the even code;
a block with a NaN or an infinity takes scale code 255 and zero elements.

Everything is float64; codes are returned one per element. Shares no code with
the GPU path.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_CODE = 255


def e2m1_encode(v) -> np.ndarray:
    """Codes of values: nearest on the grid (saturating), ties to the even code."""
    v = np.asarray(v, np.float64)
    d = np.abs(np.minimum(np.abs(v), 6.0)[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    tied = d == best
    even = tied & (np.arange(8) % 2 == 0)
    pick = np.where(tied.sum(-1) > 1, even.argmax(-1), tied.argmax(-1))
    return (pick + np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def scale_code(top) -> np.ndarray:
    """Scale codes of blocks with largest magnitude ``top`` (finite)."""
    top = np.asarray(top, np.float64)
    e = np.frexp(top)[1] - 1  # top = m 2^(e + 1), m in [1/2, 1)
    return np.where(top > 0, np.maximum(e - 2 + 127, 0), 0).astype(np.int64)


def quantize(x):
    """Rows [.., K] (K % 32 == 0) -> codes [.., K] uint8, scale codes [.., K / 32] uint8."""
    v = np.asarray(x, np.float64)
    b = v.reshape(v.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(b).all(-1)
    safe = np.where(bad[..., None], 0.0, b)
    c = scale_code(np.abs(safe).max(-1))
    q = e2m1_encode(safe / np.exp2(c - 127.0)[..., None])
    q = np.where(bad[..., None], 0, q).astype(np.uint8)
    return q.reshape(v.shape), np.where(bad, NAN_CODE, c).astype(np.uint8)


def values(codes, scales):
    """float64 values of codes [.., K] under scale codes [.., K / 32]."""
    c = np.asarray(codes, np.int64)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.exp2(np.asarray(scales, np.float64) - 127.0)
    s = np.where(np.asarray(scales) == NAN_CODE, np.nan, s)
    return (v.reshape(v.shape[:-1] + (-1, 32)) * s[..., None]).reshape(v.shape)


def pack(codes, scales):
    """(codes, scale codes) of rows [.., R, K] in the operand layout: bytes
    [.., R, 128 C] and int32 scale dwords [.., C, R, 2], C = ceil(K / 256)."""
    K = codes.shape[-1]
    C = (K + 255) // 256
    pad = [(0, 0)] * (codes.ndim - 1)
    q = np.pad(codes, pad + [(0, 256 * C - K)])
    s = np.pad(scales, pad + [(0, 8 * C - K // 32)])
    b = (q[..., 0::2] | (q[..., 1::2] << 4)).astype(np.uint8)
    s = s.reshape(s.shape[:-1] + (C, 4, 2))           # block 2 s + h of a chunk
    s = np.moveaxis(np.swapaxes(s, -1, -2), -3, -4)   # [.., C, R, h, s]
    return np.ascontiguousarray(b), np.ascontiguousarray(s).astype(np.uint8).view(np.int32)[..., 0]


def unpack(b, dwords, K):
    """The inverse of ``pack``: (codes [.., R, K], scale codes [.., R, K / 32])."""
    q = np.stack((b & 15, b >> 4), -1).reshape(b.shape[:-1] + (-1,))[..., :K]
    s = np.ascontiguousarray(dwords).view(np.uint8).reshape(dwords.shape + (4,))  # [.., C, R, h, s]
    s = np.swapaxes(np.moveaxis(s, -4, -3), -1, -2)                               # [.., R, C, s, h]
    return q, s.reshape(s.shape[:-3] + (-1,))[..., : K // 32]


def silu(g):
    return g / (1.0 + np.exp(-g))
