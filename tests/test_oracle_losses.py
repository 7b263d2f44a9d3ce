"""The oracle of the losses against automatic differentiation of their formulas, written with torch's own functions."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import losses as O


def _case(rows, vocab, seed):
    rng = np.random.default_rng(seed)
    z = 2 * rng.standard_normal((rows, vocab))
    ids = rng.integers(0, vocab, rows)
    w = rng.random(rows)
    w[::4] = 0.0
    return rng, z, torch.from_numpy(z).requires_grad_(), ids, w


def _same(got, want):
    np.testing.assert_allclose(got, want.detach().numpy() if torch.is_tensor(want) else want, rtol=1e-11, atol=1e-13)


@pytest.mark.parametrize("rows,vocab", [(1, 2), (9, 17)])
@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_token_loss(rows, vocab, scale):
    rng, z, t, ids, w = _case(rows, vocab, 1)
    if rows > 1:
        w[1] = 0.7
        ids[1] = -1
    loss = F.cross_entropy(scale * t, torch.from_numpy(ids), reduction="none", ignore_index=-1) * torch.from_numpy(w)
    got = O.token_loss(z, ids, w, scale)
    _same(got[0], loss)
    _same(got[2], torch.autograd.grad(loss.sum(), t)[0])
    lp, lse = O.logp(z, ids, scale)
    on = ids >= 0
    _same(lse[on], torch.logsumexp(scale * t, 1)[on])
    _same(-w * lp, got[0])
    g = rng.standard_normal(rows)
    _same(O.logp_bwd(z, ids, lse, g, scale), O.token_loss(z, ids, -g, scale)[2])


def test_logp_of_shards():
    rng, z, t, ids, _ = _case(8, 30, 2)
    lp, lse = O.logp(z, ids)
    parts = [O.logp(z[:, i:i + 10], ids, first=i) for i in (0, 10, 20)]
    _same(np.logaddexp.reduce([p[1] for p in parts]), lse)
    _same(sum(p[0] + p[1] for p in parts) - lse, lp)
    g = rng.standard_normal(8)
    _same(np.concatenate([O.logp_bwd(z[:, i:i + 10], ids, lse, g, first=i) for i in (0, 10, 20)], 1), O.logp_bwd(z, ids, lse, g))


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_loss(kl):
    rng, z, t, ids, w = _case(40, 11, 3)
    lp = F.log_softmax(0.8 * t, 1)[torch.arange(40), torch.from_numpy(ids)]
    old, ref = lp.detach().numpy() - 0.4 * rng.standard_normal(40), lp.detach().numpy() + 0.3 * rng.standard_normal(40)
    adv = rng.standard_normal(40)
    r, a, d = (lp - torch.from_numpy(old)).exp(), torch.from_numpy(adv), torch.from_numpy(ref) - lp
    loss = torch.from_numpy(w) * (-torch.minimum(r * a, r.clamp(0.8, 1.3) * a) + kl * (d.exp() - d - 1))
    got = O.policy_loss(z, ids, old, adv, ref, w, 0.2, 0.3, kl, 0.8)
    _same(got[0], loss)
    _same(got[1], np.where(w != 0, lp.detach().numpy(), 0))
    _same(got[2], torch.autograd.grad(loss.sum(), t)[0])


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_loss(smoothing):
    rng, z, t, ids, w = _case(30, 7, 4)
    ref, starts, pw = rng.standard_normal(30) - 2, np.array([2, 9, 9, 20, 27]), np.array([0.5, 2.0])
    lp = F.log_softmax(t, 1)[torch.arange(30), torch.from_numpy(ids)]
    gain = torch.from_numpy(w) * (lp - torch.from_numpy(ref))
    s = torch.stack([gain[a:b].sum() for a, b in zip(starts, starts[1:])])
    x = 0.3 * (s[0::2] - s[1::2]) - 0.1
    loss = -torch.from_numpy(pw) * ((1 - smoothing) * F.logsigmoid(x) + smoothing * F.logsigmoid(-x))
    got = O.preference_loss(z, ids, starts, ref, w, pw, 0.3, 0.1, smoothing)
    _same(got[0], loss)
    _same(got[1], 0.3 * s)
    _same(got[2], torch.autograd.grad(loss.sum(), t)[0])
    assert not got[2][:2].any() and not got[2][27:].any()


@pytest.mark.parametrize("rest", [False, True])
def test_distillation(rest):
    rng, z, t, _, w = _case(9, 20, 5)
    teacher = 1.5 * rng.standard_normal((9, 20))
    at = np.stack([rng.permutation(20)[:6] for _ in range(9)])
    tl = np.take_along_axis(teacher, at, 1)
    lse = torch.logsumexp(0.5 * torch.from_numpy(teacher), 1).numpy() if rest else None
    p, idx = F.softmax(0.5 * t, 1), torch.from_numpy(at)
    if rest:
        q = torch.exp(0.5 * torch.from_numpy(tl) - torch.from_numpy(lse)[:, None])
        q = torch.cat([q, 1 - q.sum(1, keepdim=True)], 1)
        p = torch.cat([p.gather(1, idx), 1 - p.gather(1, idx).sum(1, keepdim=True)], 1)
    else:
        q, p = F.softmax(0.5 * torch.from_numpy(tl), 1), p.gather(1, idx)
    loss = torch.from_numpy(w) * F.kl_div(p.log(), q, reduction="none").sum(1)
    got = O.distill_loss(z, at, tl, lse, w, 0.5)
    _same(got[0], loss)
    _same(got[1], torch.autograd.grad(loss.sum(), t)[0])
    # an entry twice: its probability twice against one column; entries that do not count change nothing
    twice = O.distill_loss(z, np.concatenate([at, at[:, :1]], 1), np.concatenate([tl, tl[:, :1]], 1), lse, w, 0.5)
    holes = O.distill_loss(z, np.concatenate([at, np.full((9, 2), -1)], 1), np.concatenate([tl, np.full((9, 2), 9.0)], 1), lse, w, 0.5)
    _same(holes[0], got[0])
    _same(holes[1], got[1])
    assert not np.allclose(twice[1], got[1])
    on = w != 0
    if not rest:
        _same(twice[1].sum(1), np.zeros(9))                        # p - q sums to nothing
    none = O.distill_loss(z, np.full((9, 3), -1), tl[:, :3], lse, w, 0.5)
    assert np.abs(none[0]).max() <= 1e-12 and np.abs(none[1]).max() <= 1e-12 and on.any()
