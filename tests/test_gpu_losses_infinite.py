"""The preference loss of pairs with a token of probability 0: a rejected sequence that cannot be, x = +inf, costs nothing, and a chosen
one costs without end."""
import numpy as np
import pytest
import torch

from loss_cases import DEV, HALF_STEP, TORCH, U, close, delta, dev, f32
from oracle import losses as O

pytestmark = pytest.mark.gpu


def _op(vocab, dtype="f32", **kw):
    from paper_2504_03662_amd.loss_ops import DevicePreferenceLoss
    return DevicePreferenceLoss(vocab, dtype, **kw)


# 8 rows and those of a launch for the pairs; rewards come from whole rows of a wavefront, a workgroup, and rows read twice
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
@pytest.mark.parametrize("rows,vocab", [(8, 50), (8, 5000), (8, 70001), (1030, 50)])
def test_a_token_of_probability_0(rows, vocab, smoothing, dtype):
    rng = np.random.default_rng(rows + vocab)
    z = torch.from_numpy(rng.standard_normal((rows, vocab))).to(TORCH[dtype]).double().numpy()
    ids = rng.integers(0, vocab, rows)
    starts = np.array([0, 2, 4, 6, 8, 8, 8], np.int32)
    z[3, ids[3]] = -np.inf                                         # rejected in the first pair
    z[4, ids[4]] = -np.inf                                         # chosen in the second; the third's sequences are empty
    pw = f32([1.5, 0.5, 2.0])
    op = _op(vocab, dtype, beta=0.5, smoothing=smoothing)
    args = torch.from_numpy(z).to(TORCH[dtype]).to(DEV), dev(ids, torch.int64), dev(starts, torch.int32)
    loss, rewards, dz = op.forward_backward(*args, pair_weights=dev(pw))
    want, want_r, want_d = O.preference_loss(z, ids, starts, None, None, pw, 0.5, 0.0, smoothing)
    inf = np.inf
    assert want[:2].tolist() == {0.0: [0.0, inf], 0.25: [inf, inf], 1.0: [inf, 0.0]}[smoothing]
    assert loss[:2].tolist() == want[:2].tolist() and abs(float(loss[2]) - 2 * np.log(2)) <= 4 * U
    assert rewards[1:3].tolist() == [-inf, -inf]
    close(rewards[[0, 3]], want_r[[0, 3]], delta(vocab) + 2 * U * np.abs(want_r[[0, 3]]), "rewards")
    # the slope by x is smoothing or smoothing - 1, without an error; p is off by 2 (|a| + 12) u + delta of itself, |a| <= 6, and a
    # token of probability 0 has the whole of the slope
    g = np.zeros(rows)
    g[:8] = 0.5 * np.repeat(pw[:2] * np.abs([smoothing, 1.0 - smoothing]), 4)
    close(dz, want_d, HALF_STEP[dtype] * np.abs(want_d) + g[:, None] * (64 * U + delta(vocab)), "dlogits")
    two = op.forward(*args, pair_weights=dev(pw))
    assert torch.equal(two[0], loss) and torch.equal(two[1], rewards)


@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
def test_log_probabilities_of_minus_infinity(smoothing):
    lp = f32([-1, -2, -np.inf, -1, -np.inf, -3, -1, -1])
    starts = np.array([0, 2, 4, 6, 8], np.int32)
    loss, rewards, g = _op(9, beta=0.5, smoothing=smoothing).pairs(dev(lp), dev(starts, torch.int32))
    want, want_r, want_g = O.pairs_loss(lp, starts, beta=0.5, smoothing=smoothing)
    assert loss.tolist() == want.tolist() == {0.0: [0.0, np.inf], 0.25: [np.inf] * 2, 1.0: [np.inf, 0.0]}[smoothing]
    assert rewards.tolist() == want_r.tolist() == [-1.5, -np.inf, -np.inf, -1.0]
    assert g.tolist() == want_g.tolist()                           # halves and quarters: exact
