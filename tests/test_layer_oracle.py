"""CPU tests of the oracle of routing, dense products and dropout: against published
vectors, differences and torch's own formulas in float64."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as O


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_philox_published_vectors(counter, key, want):
    assert tuple(O.philox(counter, key)) == want


def test_dropout_rate_and_scale():
    n, p = 40000, 0.3
    y = O.dropout_add(np.ones(n), p, 12345, 7)
    kept = float((y != 0).mean())
    assert abs(kept - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
    assert set(np.unique(y)) == {0.0, float(np.float32(1 / 0.7))}


def test_dropout_counter_wraps():
    a = O.dropout_words(16, 3, (1 << 64) - 2)
    assert np.array_equal(a[8:], O.dropout_words(8, 3, 0))


@pytest.mark.parametrize("score,norm", [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)])
def test_route_backward_against_differences(score, norm):
    r = np.random.default_rng(1)
    z, dw = r.standard_normal((5, 12)), r.standard_normal((5, 3))
    ids, _ = O.route(z, 3, score, norm=norm)

    def value(zz):
        s = np.stack([O.scores(row, score) for row in zz])
        w = np.take_along_axis(s, ids.astype(int), 1)
        return 1.7 * ((w / w.sum(1, keepdims=True) if norm else w) * dw).sum()

    got = O.route_backward(z, ids, dw, score, norm, 1.7)
    for t in range(5):
        for e in range(12):
            h = np.zeros_like(z)
            h[t, e] = 1e-6
            assert abs((value(z + h) - value(z - h)) / 2e-6 - got[t, e]) < 1e-8


def test_route_groups_bias_and_ties():
    # two groups of the same sum: the lower one; the bias moves the selection, not the weights
    z = np.array([[0.0, 2.0, 1.0, 1.0, -1.0, 3.0]])
    ids, w = O.route(z, 2, "softmax", n_group=3, topk_group=1, norm=False)
    assert ids.tolist() == [[5, 4]]
    b = np.array([5.0, 0, 0, 0, 0, 0])
    ids, w2 = O.route(z, 2, "softmax", bias=b, n_group=3, topk_group=1, norm=False)
    assert ids.tolist() == [[0, 1]]
    assert np.allclose(w2[0], O.scores(z[0], "softmax")[[0, 1]])
    ids, _ = O.route(np.zeros((1, 6)), 2, n_group=3, topk_group=1)
    assert ids.tolist() == [[0, 1]]


def test_route_with_nothing_to_select():
    z = np.array([[-np.inf] * 4, [-np.inf, 1.0, -np.inf, -np.inf], [np.nan, 1.0, 2.0, 0.0]])
    ids, w = O.route(z, 2)
    assert ids.tolist() == [[-1, -1], [1, -1], [2, 1]]
    assert np.array_equal(w[:2], [[0, 0], [1, 0]]) and np.isnan(w[2]).all()
    ids, _ = O.route(z, 2, mask=np.array([1, 0, 1]))
    assert ids[1].tolist() == [-1, -1]


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_act_against_torch(name):
    z = torch.linspace(-9, 9, 401, dtype=torch.float64, requires_grad=True)
    f = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[name]
    y = f(z)
    y.sum().backward()
    a, slope = O.act(z.detach().numpy(), name)
    assert np.allclose(a, y.detach().numpy(), atol=1e-12) and np.allclose(slope, z.grad.numpy(), atol=1e-12)


def test_act_backward_against_torch():
    r = np.random.default_rng(0)
    z, m, dy = (torch.from_numpy(r.standard_normal((7, 9))) for _ in range(3))
    z.requires_grad_(), m.requires_grad_()
    (torch.nn.functional.silu(z) * m).backward(dy)
    dz, dmul = O.act_backward(dy.numpy(), z.detach().numpy(), "silu", m.detach().numpy())
    assert np.allclose(dz, z.grad.numpy()) and np.allclose(dmul, m.grad.numpy())
