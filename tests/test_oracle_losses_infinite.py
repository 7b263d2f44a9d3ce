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


def test_shards_of_nothing():
    """Columns of -inf are none, whole shards of them too"""
    rng = np.random.default_rng(0)
    z, ids = rng.standard_normal((4, 12)), np.array([1, 5, 5, 9])
    z[0, 4:8] = z[1, 4:8] = z[2, 8:] = z[3, :8] = -np.inf
    lp, lse = O.logp(z, ids)
    parts = [O.logp(z[:, i:i + 4], ids, first=i) for i in (0, 4, 8)]
    np.testing.assert_allclose(np.logaddexp.reduce([p[1] for p in parts]), lse, rtol=1e-12)
    whole = sum(p[0] + np.where(p[1] == -np.inf, 0.0, p[1]) for p in parts) - lse
    assert whole[1] == lp[1] == -np.inf
    np.testing.assert_allclose(whole[[0, 2, 3]], lp[[0, 2, 3]], rtol=1e-12)


@pytest.mark.parametrize("rest", [False, True])
def test_distillation_without_an_entry(rest):
    z = np.array([[1.0, np.nan, -np.inf], [0.5, 0.0, 2.0]])
    loss, d = O.distill_loss(z, np.array([[-1, 3], [-1, 2]]), np.zeros((2, 2)), np.array([np.nan, 1.0]) if rest else None)
    assert loss[0] == 0 and not d[0].any() and loss[1] > 0 and d[1].all()
