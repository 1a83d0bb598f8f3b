"""CPU tests of the training oracle: losses by hand, gradients against differences."""
import numpy as np
import pytest

from oracle import train_oracle as R


def _case(seed, T, E, k, seq, masked):
    r = np.random.default_rng(seed)
    z = 2.0 * r.standard_normal((T, E))
    ids = np.argsort(-z, axis=1)[:, :k]
    mask = (r.random(T) > 0.4).astype(np.uint8) if masked else None
    return r, z, ids, mask


def test_equal_and_skewed_loads():
    E, k, T = 8, 2, 16
    ids = np.stack([np.arange(T) % E, (np.arange(T) + 1) % E], 1)
    loss, counts, live = R.balance(np.zeros((T, E)), ids)
    assert np.isclose(loss[0], 1.0) and np.isclose(loss[1], np.log(E) ** 2)
    assert counts.tolist() == [[4] * E] and live.tolist() == [T, T, 1]
    z = np.zeros((T, E))
    z[:, :2] = 50.0
    loss, counts, _ = R.balance(z, np.tile([0, 1], (T, 1)))
    assert np.isclose(loss[0], E / k)


def test_masked_rows_and_empty_groups():
    z = np.random.default_rng(0).standard_normal((9, 4))
    z[3:6] = np.nan
    ids = np.zeros((9, 1), int)
    mask = np.array([1, 1, 0, 0, 0, 0, 1, 0, 0])
    loss, counts, live = R.balance(z, ids, mask, seq=3)
    assert np.isfinite(loss).all() and live.tolist() == [2, 0, 1, 3, 2] and counts[:, 0].tolist() == [2, 0, 1]
    assert R.balance(z, ids, np.zeros(9), seq=3)[0].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("T,E,k,seq,masked", [(6, 5, 2, 0, False), (12, 8, 3, 4, True), (4, 3, 1, 1, False)])
def test_loss_gradient_against_differences(T, E, k, seq, masked):
    """ids are constants of the loss: the counts do not move with the logits."""
    r, z, ids, mask = _case(T, T, E, k, seq, masked)
    g = r.standard_normal(2)
    loss, counts, live = R.balance(z, ids, mask, seq)
    d, _ = R.gate_gradient(z, ids, counts, live, g, mask=mask, seq=seq)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            up, dn = z.copy(), z.copy()
            up[t, e] += h
            dn[t, e] -= h
            num = (R.balance(up, ids, mask, seq)[0] - R.balance(dn, ids, mask, seq)[0]) @ g / (2 * h)
            assert abs(num - d[t, e]) <= 1e-8 + 1e-6 * abs(num)


def test_gate_weight_gradient_against_differences():
    r, z, ids, _ = _case(3, 5, 7, 3, 0, False)
    dw = r.standard_normal((5, 3))

    def weights(z):
        v = np.take_along_axis(z, ids, 1)
        e = np.exp(v - v.max(1, keepdims=True))
        return e / e.sum(1, keepdims=True)

    _, counts, live = R.balance(z, ids)
    d, _ = R.gate_gradient(z, ids, counts, live, [0.0, 0.0], weights(z), dw)
    h = 1e-6
    for t in range(5):
        for e in range(7):
            up, dn = z.copy(), z.copy()
            up[t, e] += h
            dn[t, e] -= h
            num = ((weights(up) - weights(dn)) * dw).sum() / (2 * h)
            assert abs(num - d[t, e]) <= 1e-8


def test_combine_gradient_against_differences():
    r = np.random.default_rng(4)
    T, k, H = 3, 2, 4
    dest = np.array([0, 3, -1, 1, 2, -1])
    y, w, do = r.standard_normal((4, H)), r.random((T, k)), r.standard_normal((T, H))

    def out(y, w):
        o = np.zeros((T, H))
        for i, d in enumerate(dest):
            if d >= 0:
                o[i // k] += w[i // k, i % k] * y[d]
        return o

    dw, _, dy = R.combine_gradient(do, y, w, dest)
    h = 1e-6
    for i in range(T * k):
        up, dn = w.copy(), w.copy()
        up[i // k, i % k] += h
        dn[i // k, i % k] -= h
        assert abs(((out(y, up) - out(y, dn)) * do).sum() / (2 * h) - dw[i // k, i % k]) <= 1e-8
    for row, (t, j) in dy.items():
        up, dn = y.copy(), y.copy()
        up[row, 1] += h
        dn[row, 1] -= h
        assert abs(((out(up, w) - out(dn, w)) * do).sum() / (2 * h) - w[t, j] * do[t, 1]) <= 1e-8
