"""Tokens that are nearly certain, 1 - p about 1e-10 .. 1e-5: 1 - p is what the gradient at the token is made of, and it is not formed by
taking p from 1.

Rows: logits of -25 .. -23 in steps of 1/8 (numbers of both types) below the token's, and -inf within 16 columns of it, so that the 16
bytes that hold the token add nothing to its 1.  With E = exp(z - z of the token) and S the sum of E elsewhere, 1 - p = S / (1 + S).
Bounds, in u = 2^-24: E's argument is a difference without an error, rounded once as a product, 25 u; the exponential 2 u; the sums over 16
bytes 3 u; what is fp64 from there on adds 2^-46 to 1 + S at most.  expm1 4 u, the gradient by logp and the scale 4 u.  A gradient in bf16
away from the token takes log2(e) as one number of fp32, which is off by 2 u of itself: twice the argument."""
import numpy as np
import pytest
import torch

from loss_cases import DEV, HALF_STEP, TINY, TORCH, U, close, dev, f32, placed
from oracle import losses as O

pytestmark = pytest.mark.gpu

# rows, vocab, elements between rows beyond vocab, first column of the view
SIZES = [(6, 40, 0, 0), (7, 1001, 3, 1), (5, 5003, 0, 0), (4, 32768, 0, 0), (5, 33001, 7, 3), (3, 70001, 0, 0), (2, 262144, 0, 0)]


def _sure(rng, rows, vocab, dtype, scale):
    """(tensor, array, tokens, E, S by row); the tokens are at the rows' ends and in between"""
    a = rng.integers(-25 * 8, -23 * 8 + 1, (rows, vocab)) / 8
    top = 4.0 * (np.arange(rows) % 2)
    ids = rng.integers(0, vocab, rows)
    ids[0], ids[1 % rows] = 0, vocab - 1
    a[np.abs(np.arange(vocab)[None, :] - ids[:, None]) <= 16] = -np.inf
    a[np.arange(rows), ids] = 0.0
    z = (a + top[:, None]) / scale
    t = torch.from_numpy(z).to(TORCH[dtype])
    assert np.array_equal(t.double().numpy(), z)
    others = np.exp(a)
    others[np.arange(rows), ids] = 0.0
    return t, z, ids, others, others.sum(1)


def _close_gradient(dz, others, s, g, ids, dtype, scale, name):
    """dz = g scale (1 at the id - p)"""
    rows = np.arange(len(ids))
    gs = (scale * np.asarray(g, float))[:, None]
    want = -gs * others / (1 + s)[:, None]
    want[rows, ids] = gs[:, 0] * s / (1 + s)
    # elsewhere p has a second product, 1 / sum, in front of it
    steps = 48 + (50 if dtype == "bf16" else 0)
    at = np.arange(want.shape[1]) == ids[:, None]
    close(dz, want, (HALF_STEP[dtype] + steps * U) * np.abs(want) + np.abs(gs) * 2.0 ** -46 * at + TINY, name)


def _ops():
    from paper_2504_03662_amd import loss_ops
    return loss_ops


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 0.5])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_cross_entropy_and_policy(size, scale, dtype):
    rows, vocab, pad, offset = size
    t, z, ids, others, s = _sure(np.random.default_rng(vocab), rows, vocab, dtype, scale)
    view, _ = placed(t, pad, offset)
    idt, want = dev(ids, torch.int64), -np.log1p(s)
    tol = s * 30 * U + 2.0 ** -46 + U * np.abs(want)
    logp, lse = _ops().DeviceTokenLoss(vocab, dtype, scale=scale).logp(view, idt)
    close(logp, want, tol, "logp")
    loss, dz = _ops().DeviceTokenLoss(vocab, dtype, scale=scale).forward_backward(view, idt)
    close(loss, -want, tol, "loss")
    _close_gradient(dz, others, s, -np.ones(rows), ids, dtype, scale, "cross entropy")
    # r = exp(logp - old) = 1 but for 1e-5 of it: within the borders, gradient -r A
    one = torch.ones(rows, device=DEV)
    loss, logp, dz = _ops().DevicePolicyLoss(vocab, dtype, scale=scale).forward_backward(view, idt, 0 * one, one)
    close(logp, want, tol, "the policy's logp")
    _close_gradient(dz, others, s, -1 / (1 + s), ids, dtype, scale, "policy")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES + [(1100, *s[1:]) for s in SIZES[:3]], ids=str)
def test_preference(size, dtype):
    """Few rows, and as many as have a launch for their pairs"""
    rows, vocab, pad, offset = size
    t, z, ids, others, s = _sure(np.random.default_rng(vocab + 1), rows, vocab, dtype, 1.0)
    view, _ = placed(t, pad, offset)
    pairs = min(rows // 2, 3)
    starts = np.arange(2 * pairs + 1) * (1 if rows < 1000 else 170)
    beta, smoothing = 0.5, 0.25
    op = _ops().DevicePreferenceLoss(vocab, dtype, beta=beta, smoothing=smoothing)
    loss, rewards, dz = op.forward_backward(view, dev(ids, torch.int64), dev(starts, torch.int32))
    lp = -np.log1p(s)
    _, want_r, g = O.pairs_loss(lp, starts, beta=beta, smoothing=smoothing)
    sums = lambda x: np.array([x[i:j].sum() for i, j in zip(starts, starts[1:])])
    close(rewards, want_r, beta * sums(s * 30 * U + 2.0 ** -46) + U * np.abs(want_r), "rewards")
    _close_gradient(dz, others, s, g, ids, dtype, 1.0, "preference")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 0.5])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient_of_given_log_probabilities(size, scale, dtype):
    """By the log sums as they are given, rounded to fp32; the argument scale z - lse is rounded once"""
    rows, vocab, pad, offset = size
    rng = np.random.default_rng(vocab + 2)
    t, z, ids, others, s = _sure(rng, rows, vocab, dtype, scale)
    view, whole = placed(t, pad, offset)
    given, g = f32(4.0 * (np.arange(rows) % 2) + np.log1p(s)), f32(rng.standard_normal(rows))
    op = _ops().DeviceTokenLoss(vocab, dtype, scale=scale)
    args = dev(ids, torch.int64), dev(given), dev(g)
    dz = op.logp_backward(view, *args)
    gs, at = (scale * g.astype(float))[:, None], np.arange(rows)
    with np.errstate(invalid="ignore"):
        want = -gs * np.exp(scale * z - given.astype(float)[:, None])
    want[at, ids] = -gs[:, 0] * np.expm1(scale * z[at, ids] - given.astype(float))
    # arguments up to 25 + 4, rounded as a sum and as a product: 58 u; exp2 and the products in front of it 8 u
    steps = 66 + (58 if dtype == "bf16" else 0)
    close(dz, want, (HALF_STEP[dtype] + steps * U) * np.abs(want) + TINY, "dlogits")
    inside = op.logp_backward(view, *args, out=view)
    assert inside is view and torch.equal(inside, dz)


@pytest.mark.parametrize("vocab", [1001, 5003])
def test_preference_over_the_logits(vocab):
    rows = 12
    t, _, ids, _, _ = _sure(np.random.default_rng(3), rows, vocab, "f32", 1.0)
    op = _ops().DevicePreferenceLoss(vocab, "f32")
    z, ids, starts = t.to(DEV), dev(ids, torch.int64), dev([0, 3, 6, 9, 12], torch.int32)
    want = op.forward_backward(z, ids, starts)
    got = op.forward_backward(z, ids, starts, out=z)
    assert got[2] is z and all(torch.equal(a, b) for a, b in zip(got, want))
