"""CPU tests of the MXFP4 oracle: the grid, rounding, scales and layout."""
import numpy as np
import pytest

from oracle import mx4_oracle as Q


def test_grid_and_ties():
    v = np.array([0.0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 6.0, 7.5, -0.25, -0.75, -5.0])
    want = np.array([0.0, 0.0, 0.5, 1.0, 0.5, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, 6.0, -0.0, -1.0, -4.0])
    q = Q.e2m1_encode(v)
    got = Q.GRID[q & 7] * np.where(q & 8, -1.0, 1.0)
    assert np.array_equal(got, want) and np.array_equal(np.signbit(got), np.signbit(want))
    codes = np.arange(16)
    back = Q.e2m1_encode(Q.GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0))
    assert np.array_equal(back, codes)


@pytest.mark.parametrize("top,code", [(0.0, 0), (1.0, 125), (6.0, 127), (7.9, 127), (8.0, 128), (0.999, 124),
                                      (2.0 ** -126, 0), (2.0 ** -125, 0), (2.0 ** -124, 1), (1e-45, 0),
                                      (float(np.finfo(np.float32).max), 252)])
def test_scale_codes(top, code):
    assert Q.scale_code(top) == code


def test_quantise_error_and_idempotence():
    r = np.random.default_rng(0)
    x = (r.standard_normal((7, 288)) * np.exp(2.0 * r.standard_normal((7, 1)))).astype(np.float32)
    q, s = Q.quantize(x)
    v = Q.values(q, s)
    scale = np.repeat(np.exp2(s.astype(float) - 127), 32, axis=1)
    # between grid points at most 2 apart, or clamped from below 8
    assert np.all(np.abs(v - x) <= np.where(np.abs(x) > 6 * scale, 2.0, 1.0) * scale)
    q2, s2 = Q.quantize(v)
    assert np.array_equal(Q.values(q2, s2), v)


def test_bad_blocks_are_nan():
    x = np.ones((1, 96), np.float32)
    x[0, 3], x[0, 70] = np.nan, -np.inf
    q, s = Q.quantize(x)
    assert s.tolist() == [[255, 125, 255]] and not q[0, :32].any() and not q[0, 64:].any()
    v = Q.values(q, s)
    assert np.isnan(v[0, :32]).all() and (v[0, 32:64] == 1.0).all() and np.isnan(v[0, 64:]).all()


@pytest.mark.parametrize("shape", [(3, 32), (5, 256), (2, 4, 288), (1, 1024)])
def test_layout_round_trip(shape):
    r = np.random.default_rng(1)
    q = r.integers(0, 16, shape).astype(np.uint8)
    s = r.integers(0, 255, shape[:-1] + (shape[-1] // 32,)).astype(np.uint8)
    b, d = Q.pack(q, s)
    C = (shape[-1] + 255) // 256
    assert b.shape == shape[:-1] + (128 * C,) and d.shape == shape[:-2] + (C, shape[-2], 2)
    q2, s2 = Q.unpack(b, d, shape[-1])
    assert np.array_equal(q, q2) and np.array_equal(s, s2)


def test_layout_by_definition():
    q = np.arange(256, dtype=np.uint8)[None] % 16
    s = (np.arange(8, dtype=np.uint8) + 100)[None]
    b, d = Q.pack(q, s)
    assert b[0, 5] == (10 | 11 << 4)
    w = d.view(np.uint32)[0, 0]
    for h in range(2):
        for k in range(4):
            assert (int(w[h]) >> (8 * k)) & 255 == 100 + 2 * k + h
