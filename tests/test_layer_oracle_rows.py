"""CPU test of the routing gradient's oracle on tokens without an expert."""
import numpy as np
import pytest

from oracle import layer_oracle as O


@pytest.mark.parametrize("score,norm", [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)])
def test_tokens_without_an_expert_have_no_gradient(score, norm):
    z = np.zeros((5, 6), np.float32)
    z[0, 2], z[1, 2], z[2, 2], z[3] = np.nan, np.inf, -np.inf, np.nan
    ids = np.full((5, 2), -1, np.int32)
    ids[1] = 6
    with np.errstate(invalid="ignore"):
        got = O.route_backward(z, ids, np.full((5, 2), np.nan), score, norm, 2.5)
    assert np.array_equal(got, np.zeros((5, 6)))
