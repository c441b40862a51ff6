"""The float64 definitions of the losses where a probability is zero, against values by hand."""
import numpy as np
import pytest

from oracle import losses


@pytest.mark.parametrize("row,eps,want", [(0, 0.0, np.inf), (1, 0.0, 0.0), (0, 0.1, np.inf), (1, 0.1, np.inf), (0, 1.0, 0.0), (1, 1.0, np.inf)])
def test_an_infinite_margin(row, eps, want):
    """-(1 - eps) log sigmoid(z) - eps log sigmoid(-z) for z = -infinity (a token of probability zero in the preferred sequence) and +infinity (in the other)."""
    x = np.zeros((2, 3))
    x[row, 1] = -np.inf
    out = losses.preference_loss(x, [1, 1], [0, 1, 2], 0.5, eps)
    assert out["loss"] == want and out["z"][0] == (-np.inf if row == 0 else np.inf) and np.isfinite(out["grad"]).all()
