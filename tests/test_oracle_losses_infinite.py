"""The oracle of the losses where a log probability is -inf"""
import numpy as np
import pytest

from oracle import losses as O


@pytest.mark.parametrize("smoothing,want", [(0.0, [0.0, np.inf]), (0.25, [np.inf, np.inf]), (1.0, [np.inf, 0.0])])
def test_pairs(smoothing, want):
    """-log sigmoid(inf) = 0, and a part of weight 0 is none"""
    lp = np.array([-1.0, -np.inf, -np.inf, -1.0])
    loss, rewards, g = O.pairs_loss(lp, np.arange(5), beta=0.5, smoothing=smoothing)
    assert loss.tolist() == want and rewards.tolist() == [-0.5, -np.inf, -np.inf, -0.5]
    assert g.tolist() == [0.5 * smoothing, -0.5 * smoothing, 0.5 * (smoothing - 1), -0.5 * (smoothing - 1)]
