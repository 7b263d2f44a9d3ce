"""Sums of the losses that fp32 would lose: rewards of long sequences whose terms nearly cancel, and the divergence from a sure teacher.
Rows and bounds as in test_gpu_losses_sure_tokens: a log probability is off by S 30 u + 2^-46 before it is rounded."""
import numpy as np
import pytest
import torch

from loss_cases import DEV, U, close, dev, f32, placed
from test_gpu_losses_sure_tokens import SIZES, _sure

pytestmark = pytest.mark.gpu


def _ops():
    from paper_2504_03662_amd import loss_ops
    return loss_ops


# How far fp64 sums of up to 1024 terms near 1024 may be off: each term is rounded, and 256 threads add up to 4 of one sign, 1024 + ... + 4096;
# where neighbours are joined they cancel
OF_SUMS = 1024 * (1024 + 256 * 10) * 2.0 ** -53


def _rewards(lp, ref, starts):
    """Sums of lp - ref"""
    return np.array([np.sum(lp[i:j].astype(np.longdouble) - ref[i:j]) for i, j in zip(starts, starts[1:])]).astype(float)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1000, 1001), (2000, 1001), (1024, 5003)])
def test_rewards(rows, vocab, dtype):
    """References of +-1024 by turns; up to 1024 rows the gradient's workgroups add the pairs up, beyond that a launch does"""
    t, _, ids, _, s = _sure(np.random.default_rng(rows), rows, vocab, dtype, 1.0)
    ref = np.where(np.arange(rows) % 2, -1024.0, 1024.0)
    starts = np.array([0, rows // 4 * 2, rows])
    starts[1] -= starts[1] % 2
    op = _ops().DevicePreferenceLoss(vocab, dtype, beta=0.5)
    args = t.to(DEV), dev(ids, torch.int64), dev(starts, torch.int32), dev(ref)
    want = _rewards(-np.log1p(s), ref, starts)
    tol = np.array([s[i:j].sum() * 30 * U + (j - i) * 2.0 ** -46 for i, j in zip(starts, starts[1:])]) + OF_SUMS
    for rewards in (op.forward_backward(*args)[1], op.forward(*args)[1]):
        close(rewards, 0.5 * want, 0.5 * tol + U * np.abs(0.5 * want), "rewards")


def test_rewards_of_given_log_probabilities():
    rng = np.random.default_rng(1)
    lp = f32(-1e-4 * rng.random(2000))
    ref = np.where(np.arange(2000) % 2, -1024.0, 1024.0)
    starts = np.array([0, 1024, 2000])
    rewards = _ops().DevicePreferenceLoss(9, beta=0.5).pairs(dev(lp), dev(starts, torch.int32), dev(ref))[1]
    want = _rewards(lp, ref, starts)
    close(rewards, 0.5 * want, 0.5 * OF_SUMS + U * np.abs(0.5 * want), "rewards")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_divergence_from_a_sure_teacher(size, rest, dtype):
    """One entry with q = 1: the loss is -logp"""
    rows, vocab, pad, offset = size
    t, z, ids, _, s = _sure(np.random.default_rng(vocab + 4), rows, vocab, dtype, 1.0)
    view, _ = placed(t, pad, offset)
    teacher = f32(np.arange(rows) % 3)
    loss = _ops().DeviceDistillation(vocab, dtype).forward(view, dev(ids[:, None], torch.int64), dev(teacher[:, None]),
                                                           dev(teacher) if rest else None)
    # z (up to 4) is added to the log sum and taken off again in fp64
    close(loss, np.log1p(s), s * 30 * U + 2.0 ** -46 + U * s, "loss")
