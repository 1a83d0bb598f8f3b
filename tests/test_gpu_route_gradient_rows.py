"""GPU tests of the routing gradient's rows that have no expert, and of logits that are not
finite.

A slot whose id is outside the experts adds nothing; a token of such slots alone (a masked or
padded row) therefore has the gradient 0 whatever its logits and dw hold, and leaves an
accumulated gradient's bits as they are (x + 0 is x). Comparisons are exact.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMS = [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)]
NOT_FINITE = [np.nan, np.inf, -np.inf]


def up(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


@pytest.mark.parametrize("E,k", [(1, 1), (8, 2), (60, 4), (65, 3), (160, 6), (256, 16)])
@pytest.mark.parametrize("score,norm", FORMS)
def test_rows_without_an_expert(E, k, score, norm):
    print("CASE route gradient rows", E, k, score, norm, flush=True)
    r = np.random.default_rng(E + k)
    T = 39
    z = r.standard_normal((T, E)).astype(np.float32)
    ids = np.argsort(r.random((T, E)), 1)[:, :k].astype(np.int32)
    dw = r.standard_normal((T, k)).astype(np.float32)
    clean = moe.moe_route_backward(up(z), up(ids, torch.int32), up(dw), score=score, norm=norm, scale=1.5)
    empty = np.arange(1, T, 2)
    for i, t in enumerate(empty):
        ids[t] = [-1, E, np.iinfo(np.int32).min, np.iinfo(np.int32).max][i % 4]
        if i % 5 < 3:
            z[t, r.integers(0, E)] = NOT_FINITE[i % 5]
        elif i % 5 == 3:
            z[t] = NOT_FINITE[i % 3]
        dw[t] = NOT_FINITE[i % 3]
    rest = np.arange(0, T, 2)
    zz, ii, dd = up(z), up(ids, torch.int32), up(dw)
    got = moe.moe_route_backward(zz, ii, dd, score=score, norm=norm, scale=1.5)
    assert (got[empty] == 0).all(), got[empty]
    assert torch.equal(got[rest], clean[rest])
    base = torch.randn((T, E), device=DEV)
    acc = moe.moe_route_backward(zz, ii, dd, score=score, norm=norm, scale=1.5, dlogits=base.clone(), accumulate=True)
    assert torch.equal(acc[empty], base[empty])
    assert torch.equal(acc[rest], base[rest] + clean[rest])


@pytest.mark.parametrize("score,norm", FORMS)
def test_rows_with_an_expert_show_their_nan(score, norm):
    """What is NaN is the formula's: the whole row of a softmax by itself, otherwise the selected experts'."""
    print("CASE route gradient NaN", score, norm, flush=True)
    r = np.random.default_rng(1)
    T, E, k = 6, 24, 3
    z = r.standard_normal((T, E)).astype(np.float32)
    ids = np.tile(np.array([3, 11, 20], np.int32), (T, 1))
    dw = r.standard_normal((T, k)).astype(np.float32)
    z[1, 11] = np.nan  # a selected one
    z[2, 5] = np.nan   # another
    z[3, 5] = -np.inf
    z[4, 5] = np.nan
    ids[4, 1:] = -1
    with np.errstate(invalid="ignore"):
        want = O.route_backward(z, ids, dw, score, norm, 1.5)
    got = moe.moe_route_backward(up(z), up(ids, torch.int32), up(dw), score=score, norm=norm, scale=1.5).cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert not np.isnan(got[[0, 3, 5]]).any()
