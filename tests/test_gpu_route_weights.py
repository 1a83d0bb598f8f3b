"""GPU tests of how exact moe_route's weights are, whichever kernel a grouping takes.

Bound: a weight is computed in 64 bits and rounded to fp32 once, so it is off by u = 2^-24 of
its value at most, or by half of fp32's least value, 2^-150. The 64-bit arithmetic of both
sides has some hundred steps at most of 2^-53 each, of arguments up to 800: below 2^-36 of the
value, which is 2^-12 u.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def check(z, k, **kw):
    put = {n: torch.from_numpy(v).to(DEV) if isinstance(v, np.ndarray) else v for n, v in kw.items()}
    ids, w = moe.moe_route(torch.from_numpy(z).to(DEV), k, **put)
    want_ids, want = O.route(z, k, **kw)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    err = np.abs(w.cpu().numpy().astype(np.float64) - want)
    tol = (1 + 2.0 ** -12) * U * np.abs(want) + 2.0 ** -150
    wrong = np.argwhere(~(err <= tol))
    assert wrong.size == 0, (float((err / (U * np.abs(want) + 2.0 ** -150)).max()), len(wrong), wrong[:3])


# whole lanes a group or one group, and groupings that are neither
CONFIGS = [(8, 2, 1, 1), (1, 1, 1, 1), (60, 4, 1, 1), (128, 8, 8, 3), (160, 6, 8, 3), (192, 9, 2, 1), (250, 16, 1, 1), (256, 8, 8, 4),
           (256, 16, 1, 1), (60, 4, 5, 2), (96, 6, 8, 3), (65, 3, 13, 4), (256, 8, 128, 20)]


@pytest.mark.parametrize("E,k,G,g", CONFIGS)
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("norm", [True, False])
def test_one_rounding(E, k, G, g, score, norm):
    print("CASE route weights", E, k, G, g, score, norm, flush=True)
    r = np.random.default_rng(E * 31 + k)
    for spread in (0.01, 1.0, 4.0, 40.0):
        z = (spread * r.standard_normal((200, E))).astype(np.float32)
        z[7] -= 300.0
        z[8] += 50.0
        b = (0.2 * r.standard_normal(E)).astype(np.float32)
        check(z, k, score=score, n_group=G, topk_group=g, norm=norm, scale=2.5, bias=b if spread != 1.0 else None,
              mask=(r.random(200) < 0.9).astype(np.uint8))


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("G,g", [(1, 1), (8, 3), (3, 2)])
def test_one_rounding_of_rows_at_their_limits(score, norm, G, g):
    """Equal logits, rows of few finite ones, the ends of fp32's exponential."""
    print("CASE route weights limits", score, norm, G, g, flush=True)
    r = np.random.default_rng(2)
    E, k = 48 if G == 3 else 128, 8
    z = r.standard_normal((24, E)).astype(np.float32)
    z[0] = 0.25
    z[1] = -np.inf
    z[1, 7] = 3.0
    z[2, 5:] = -np.inf
    z[3] = np.finfo(np.float32).min
    z[4] = -800.0
    z[5] = -100.0 - np.arange(E)
    z[6] = 88.0 - 8.0 * np.arange(E)
    z[7] = np.finfo(np.float32).max
    z[8] = -87.5
    z[9] = np.nextafter(np.float32(1), np.float32(2))
    z[9, ::2] = 1.0
    z[10, 0], z[10, 1] = 88.0, -88.0
    with np.errstate(over="ignore"):
        check(z, k, score=score, n_group=G, topk_group=g, norm=norm, scale=1.0)
        check(z, k, score=score, n_group=G, topk_group=g, norm=norm, scale=16.0)
