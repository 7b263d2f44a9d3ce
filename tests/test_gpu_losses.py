"""The losses of logits on the GPU against their definition in 64 bits, at the sizes, layouts and values where they can go wrong."""
import numpy as np
import pytest
import torch

from loss_cases import DEV, HALF_STEP, TINY, TORCH, U, close, delta, dev, f32, gradient_bound, logits, placed
from oracle import losses as O

pytestmark = pytest.mark.gpu

# rows, vocab, elements between rows beyond vocab, first column of the view
SIZES = [(1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 0, 0), (4, 8, 0, 0), (6, 9, 3, 1), (3, 63, 0, 0), (70, 100, 5, 3), (33, 1001, 0, 0), (5, 2048, 0, 0),
         (9, 2049, 7, 7), (4, 4099, 0, 0), (3, 16384, 8, 8), (3, 16391, 0, 0), (2, 32768, 0, 0), (3, 32771, 1, 0), (2, 65536, 0, 0), (2, 65543, 0, 0),
         (2, 131072, 0, 0), (2, 131081, 0, 0), (1, 262144, 0, 0), (1, 524288, 0, 0), (300, 520, 0, 0), (257, 20001, 0, 0)]


@pytest.fixture(autouse=True)
def seed():
    torch.manual_seed(0)


def _ops():
    from paper_2504_03662_amd import loss_ops
    return loss_ops


def _untouched(whole, vocab, offset):
    rest = torch.ones(whole.shape[1], dtype=torch.bool, device=DEV)
    rest[offset:offset + vocab] = False
    assert bool((whole[:, rest] == 77).all())


def _inputs(size, dtype, seed):
    rows, vocab, pad, offset = size
    rng = np.random.default_rng(seed)
    t, z = logits(rng, rows, vocab, dtype)
    view, whole = placed(t, pad, offset)
    ids = rng.integers(0, vocab, rows)
    w = f32(rng.random(rows) + 0.5)
    w[rng.random(rows) < 0.2] = 0.0
    return rng, z, view, whole, ids, w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_token_loss_and_logp(size, dtype):
    rows, vocab, pad, offset = size
    rng, z, view, whole, ids, w = _inputs(size, dtype, rows + vocab)
    ids[rng.random(rows) < 0.15] = -1
    scale = [1.0, 0.5, 1.25][vocab % 3]
    op = _ops().DeviceTokenLoss(vocab, dtype, scale=scale)
    idt = torch.int32 if rows % 2 else torch.int64
    logp, lse = op.logp(view, dev(ids, idt))
    want, want_lse = O.logp(z, ids, scale)
    tol = delta(vocab) + U * (1 + np.abs(want_lse))
    close(lse, want_lse, tol, "lse")
    close(logp, want, tol + U * np.abs(want), "logp")

    loss, dz = op.forward_backward(view, dev(ids, idt), dev(w))
    want, lp, want_d = O.token_loss(z, ids, w, scale)
    close(loss, want, w * delta(vocab) + U * np.abs(want), "loss")
    close(dz, want_d, gradient_bound(want_d, z, scale, w, ids, dtype), "dlogits")
    assert torch.equal(op.forward(view, dev(ids, idt), dev(w)), loss)

    g = f32(rng.standard_normal(rows))
    g[rng.random(rows) < 0.2] = 0.0
    given = f32(want_lse + np.log(3.0))                            # as of three shards
    want_d = O.logp_bwd(z, ids, given, g, scale)
    out, out_whole = placed(torch.zeros(rows, vocab, dtype=TORCH[dtype]), pad, offset)
    got = op.logp_backward(view, dev(ids, idt), dev(given), dev(g), out=out)
    assert got is out
    _untouched(out_whole, vocab, offset)
    close(out, want_d, gradient_bound(want_d, z, scale, g, ids, dtype, lse=given.astype(float)), "dlogits of dlogp")
    _untouched(whole, vocab, offset)


def _policy_inputs(rng, z, ids, scale, low, high):
    """Ratios on both sides of the borders, none within a thousandth of one"""
    lp = O.token_loss(z, ids, None, scale)[1]
    gain = 0.3 * rng.standard_normal(len(ids))
    for border in (np.log1p(high), np.log1p(-low)):
        gain = np.where(np.abs(gain - border) < 1e-3, border + 2e-3, gain)
    adv = f32(rng.standard_normal(len(ids)))
    adv[::5] = 0.0
    return f32(lp - gain), adv, f32(lp + 0.4 * rng.standard_normal(len(ids)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kl", [0.0, 0.1])
@pytest.mark.parametrize("size", [s for s in SIZES if s[0] > 1], ids=str)
def test_policy_loss(size, kl, dtype):
    rows, vocab, pad, offset = size
    rng, z, view, whole, ids, w = _inputs(size, dtype, 7 * rows + vocab)
    scale, low, high = 1.0 if vocab % 2 else 0.75, 0.2, 0.25
    old, adv, ref = _policy_inputs(rng, z, ids, scale, low, high)
    ids[rng.random(rows) < 0.1] = -1
    op = _ops().DevicePolicyLoss(vocab, dtype, clip_low=low, clip_high=high, kl=kl, scale=scale)
    args = dev(ids, torch.int64), dev(old), dev(adv)
    loss, logp, dz = op.forward_backward(view, *args, ref_logp=dev(ref) if kl else None, weights=dev(w))
    want, lp, want_d = O.policy_loss(z, ids, old, adv, ref, w, low, high, kl, scale)
    # the borders are fp32: 0.2 is off by u / 4 of 1
    on = np.where((ids == -1) | (w == 0), 0.0, w)
    r, d = np.exp(np.where(on > 0, lp - old, 0)), np.where(on > 0, ref - lp, 0)
    size_of = on * (r * np.abs(adv) + kl * (np.exp(d) + 1 + np.abs(d)))
    slope_error = size_of * (delta(vocab) + 8 * U)
    close(logp, lp, delta(vocab) + 2 * U * np.abs(lp), "logp")
    close(loss, want, slope_error + 2 * U * np.abs(want), "loss")
    close(dz, want_d, gradient_bound(want_d, z, scale, size_of, ids, dtype, extra=slope_error), "dlogits")
    two = op.forward(view, *args, ref_logp=dev(ref) if kl else None, weights=dev(w))
    assert torch.equal(two[0], loss) and torch.equal(two[1], logp)


def _starts(rng, rows, pairs):
    """Ragged sequences, some empty, rows before the first and behind the last"""
    return np.sort(rng.integers(rows // 10, rows - rows // 10 + 1, 2 * pairs + 1)).astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,size", [(1, (2, 9, 0, 0)), (1, (40, 100, 5, 3)), (4, (70, 1001, 0, 0)), (30, (45, 65, 0, 0)), (3, (130, 16391, 0, 0)),
                                        (2, (1000, 33, 0, 0)), (1, (2, 131081, 0, 0)), (1, (2, 262144, 0, 0)), (700, (3001, 17, 0, 0))], ids=str)
def test_preference_loss(pairs, size, dtype):
    rows, vocab, pad, offset = size
    rng, z, view, whole, ids, w = _inputs(size, dtype, 3 * rows + vocab)
    starts = _starts(rng, rows, pairs)
    ids[rng.random(rows) < 0.1] = -1
    scale, beta, margin, smoothing = 0.8, 0.2, 0.3, 0.05 * (pairs % 3)
    ref = f32(O.token_loss(z, ids, None, scale)[1] + 0.2 * rng.standard_normal(rows)) if pairs != 4 else None
    pw = f32(rng.random(pairs) + 0.5)
    pw[rng.random(pairs) < 0.1] = 0.0
    op = _ops().DevicePreferenceLoss(vocab, dtype, beta=beta, margin=margin, smoothing=smoothing, scale=scale)
    kw = dict(ref_logp=dev(ref), weights=dev(w), pair_weights=dev(pw))
    args = dev(ids, torch.int64), dev(starts, torch.int32)
    loss, rewards, dz = op.forward_backward(view, *args, **kw)
    want, want_r, want_d = O.preference_loss(z, ids, starts, ref, w, pw, beta, margin, smoothing, scale)
    on = np.where(ids == -1, 0.0, w)
    total = np.concatenate([[0.0], np.cumsum(on)])
    error = beta * delta(vocab) * np.diff(total[starts])           # of a reward
    close(rewards, want_r, error + 2 * U * np.abs(want_r), "rewards")
    pair_error = error[0::2] + error[1::2] + 4 * U                 # of x: margin and smoothing are fp32
    close(loss, want, pw * pair_error * 2 + 2 * U * np.abs(want), "loss")
    seq = np.searchsorted(starts[1:], np.arange(rows), side="right")
    of = np.where((seq < 2 * pairs) & (np.arange(rows) >= starts[0]), seq // 2, -1)
    g = np.where(of >= 0, on * beta * pw[of], 0.0)
    extra = g * np.where(of >= 0, pair_error[of], 0.0)
    close(dz, want_d, gradient_bound(want_d, z, scale, g, ids, dtype, extra=extra), "dlogits")
    two = op.forward(view, *args, **kw)
    assert torch.equal(two[0], loss) and torch.equal(two[1], rewards)


def test_pairs_from_log_probabilities():
    rng = np.random.default_rng(5)
    for n, pairs in ((1, 1), (50, 3), (5000, 40), (9000, 1)):
        lp, ref, w, starts = f32(-3 * rng.random(n)), f32(-3 * rng.random(n)), f32(rng.random(n) > 0.3), _starts(rng, n, pairs)
        op = _ops().DevicePreferenceLoss(10, beta=0.05, smoothing=0.1)
        got = op.pairs(dev(lp), dev(starts, torch.int32), dev(ref), dev(w))
        want = O.pairs_loss(lp, starts, ref, w, None, 0.05, 0.0, 0.1)
        for x, y, name in zip(got, want, ("loss", "rewards", "dlogp")):
            # beta and smoothing are fp32; the sums are 64 bits
            close(x, y, 4 * U * np.abs(y) + 4 * U * (0.05 if name == "dlogp" else np.abs(want[1]).max() + 1), name)


def _teacher(rng, z, top, kind, dtype):
    """(ids, logits as numbers of the type) of the student's columns with noise"""
    rows, vocab = z.shape
    t = z + rng.standard_normal(z.shape)
    at = np.argsort(-t, 1)[:, :top]
    tl = np.take_along_axis(t, at, 1)
    lse = np.array([O.softmax(0.5 * r)[1] for r in t])
    if kind == "holes" and top > 1:
        at[rng.random(at.shape) < 0.3] = -1
        at[0] = -1                                                 # a row without an entry
        at[-1, 0] = vocab + 5
    if kind == "twice" and top > 2:
        at[:, 2] = at[:, 0]
        at[::2, 1] = at[::2, 0]
    return at, torch.from_numpy(tl).to(TORCH[dtype]), f32(lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["plain", "holes", "twice"])
@pytest.mark.parametrize("top,size", [(1, (1, 1, 0, 0)), (1, (3, 7, 0, 0)), (9, (6, 9, 3, 1)), (5, (70, 100, 5, 3)), (64, (33, 1001, 0, 0)),
                                      (1000, (2, 2049, 7, 7)), (63, (3, 16391, 0, 0)), (65, (2, 32768, 0, 0)), (256, (2, 65543, 0, 0)),
                                      (1024, (2, 131081, 0, 0)), (3, (1, 262144, 0, 0)), (17, (1, 524288, 0, 0))], ids=str)
def test_distillation(top, size, kind, rest, dtype):
    rows, vocab, pad, offset = size
    rng, z, view, whole, _, w = _inputs(size, dtype, 5 * rows + vocab + top)
    at, tl, tlse = _teacher(rng, z, top, kind, "f32" if rest else dtype)
    scale = 0.5
    op = _ops().DeviceDistillation(vocab, dtype, scale=scale)
    lse = tlse if rest else None
    idt = torch.int32 if top % 2 else torch.int64
    args = dev(at, idt), tl.to(DEV)
    loss, dz = op.forward_backward(view, *args, top_lse=dev(lse), weights=dev(w))
    want, want_d = O.distill_loss(z, at, tl.double().numpy(), lse, w, scale)
    # two log sums in the loss; q itself is rounded once
    ok = (at >= 0) & (at < vocab)
    logq = scale * tl.double().numpy() - (tlse.astype(float)[:, None] if rest else 0.0)
    q = np.where(ok, np.exp(logq), 0.0)
    if not rest:
        q = q / np.maximum(q.sum(1, keepdims=True), 1e-300)
    r = np.maximum(0, 1 - q.sum(1)) if rest else np.zeros(rows)
    mass = (q.sum(1) + r)[:, None]
    close(loss, want, w * (2 * mass[:, 0] * (delta(vocab) + 4 * U)) + 2 * U * np.abs(want), "loss")
    a = scale * z
    p = np.exp(a - np.array([O.softmax(x)[1] for x in a])[:, None])
    entry, teacher = np.zeros(z.shape, bool), np.zeros(z.shape)
    for i in range(rows):
        entry[i, at[i][ok[i]]] = True
        np.add.at(teacher[i], at[i][ok[i]], q[i][ok[i]])
    others = np.where(entry, 0.0, p)
    teacher += r[:, None] * others / np.maximum(others.sum(1, keepdims=True), 1e-300)
    error = (mass * p + teacher) * (2 * np.abs(a - a.max(1, keepdims=True)) * U + 24 * U + 2 * delta(vocab))
    close(dz, want_d, HALF_STEP[dtype] * np.abs(want_d) + scale * w[:, None] * error + TINY, "dlogits")
    assert torch.equal(op.forward(view, *args, top_lse=dev(lse), weights=dev(w)), loss)
    _untouched(whole, vocab, offset)


def _calls(vocab, dtype, rows, seed=0):
    """name -> call(logits, out) of every operator with a gradient, for any logits of these sizes"""
    ops, rng = _ops(), np.random.default_rng(seed)
    ids = dev(rng.integers(0, vocab, rows), torch.int64)
    r = lambda: dev(rng.standard_normal(rows))
    w, old, adv, ref, lse, g = dev(rng.random(rows) + 0.1), r() - 5, r(), r() - 5, r() + 9, r()
    starts = dev([0, rows // 3, rows], torch.int32)
    starts = torch.cat([starts, starts[-1:].clone(), starts[-1:]])
    k = min(7, vocab)
    at = dev(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]), torch.int64)
    tl = dev(rng.standard_normal((rows, k)))
    token, policy = ops.DeviceTokenLoss(vocab, dtype), ops.DevicePolicyLoss(vocab, dtype, kl=0.1)
    pref, distill = ops.DevicePreferenceLoss(vocab, dtype), ops.DeviceDistillation(vocab, dtype)
    return dict(token=lambda z, out=None: token.forward_backward(z, ids, w, out=out),
                logp=lambda z, out=None: (*token.logp(z, ids), token.logp_backward(z, ids, lse, g, out=out)),
                policy=lambda z, out=None: policy.forward_backward(z, ids, old, adv, ref, w, out=out),
                preference=lambda z, out=None: pref.forward_backward(z, ids, starts, ref, w, out=out),
                distill=lambda z, out=None: distill.forward_backward(z, at, tl, weights=w, out=out),
                rest=lambda z, out=None: distill.forward_backward(z, at, tl, lse, w, out=out))


NAMES = ["token", "logp", "policy", "preference", "distill", "rest"]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype,vocab", [("bf16", 1001), ("f32", 1001), ("bf16", 20000), ("bf16", 140001), ("f32", 70001)])
def test_over_the_logits_and_otherwise_laid_out(name, dtype, vocab):
    rows = 11
    call = _calls(vocab, dtype, rows)[name]
    z = (3 * torch.randn(rows, vocab, device=DEV)).to(TORCH[dtype])
    want = call(z)
    assert _same(call(z), want)                                    # the same bits
    # rows that begin at another element of 16 bytes than the logits'
    for offset in (1, 3):
        out, whole = placed(torch.zeros(rows, vocab, dtype=z.dtype), 5, offset)
        assert _same(call(z, out), want)
        _untouched(whole, vocab, offset)
    # logits that do; their sums come in another order
    view, whole = placed(z, 7, 2)
    got = call(view)
    lie = [(t.data_ptr() % 16, t.stride(0) * t.element_size() % 16) for t in (view, got[-1])]
    assert lie[0] == lie[1]
    # Each of the two is off by delta in its log sums: by delta of itself where it has a factor exp(logp - old), by up to delta times
    # the sum of weights (below 11, or 0.1 x 11 for pairs) where it is a loss
    for x, y in zip(got, want):
        bound = 4 * (HALF_STEP[dtype] + delta(vocab)) * float(y.double().abs().max()) + 22 * delta(vocab) * (x is not got[-1])
        assert float((x.double() - y.double()).abs().max()) <= bound
    inside = z.clone()
    got = call(inside, inside)
    assert got[-1] is inside and _same(got, want)
    # in three dimensions
    shaped = z[:10].view(2, 5, vocab)
    if name == "token":
        op = _ops().DeviceTokenLoss(vocab, dtype)
        ids = torch.randint(0, vocab, (2, 5), device=DEV)
        a, b = op.forward_backward(shaped, ids), op.forward_backward(z[:10], ids.view(-1))
        assert a[1].shape == shaped.shape and torch.equal(a[1].view(10, vocab), b[1]) and torch.equal(a[0].view(-1), b[0])


@pytest.mark.parametrize("dtype,vocab", [("bf16", 1001), ("f32", 1001), ("bf16", 20000), ("bf16", 140001), ("f32", 70001)])
def test_rows_that_do_not_count_are_not_looked_at(dtype, vocab):
    rows = 12
    ops, rng = _ops(), np.random.default_rng(1)
    z = (3 * torch.randn(rows, vocab, device=DEV)).to(TORCH[dtype])
    ids = torch.randint(0, vocab, (rows,), device=DEV)
    r = lambda: torch.randn(rows, device=DEV)
    w, old, adv, ref = torch.rand(rows, device=DEV) + 0.1, r(), r(), r()
    out_by_id, out_by_weight = [2, 7], [4, 11]
    w[out_by_weight] = 0.0
    ids[out_by_id] = -1
    at, tl = torch.randint(0, vocab, (rows, 5), device=DEV), torch.randn(rows, 5, device=DEV)
    starts = dev([0, 5, 10], torch.int32)                          # rows 10 and 11 are of no sequence
    bad = lambda t: [x.index_fill(0, torch.tensor(out_by_id + out_by_weight, device=DEV), float("nan")) if x.is_floating_point() and x is not w
                     else x for x in t]
    token, policy = ops.DeviceTokenLoss(vocab, dtype), ops.DevicePolicyLoss(vocab, dtype, kl=0.1)
    pref, distill = ops.DevicePreferenceLoss(vocab, dtype), ops.DeviceDistillation(vocab, dtype)
    zeros = out_by_id + out_by_weight
    for call, args, gone in ((lambda z, *a: token.forward_backward(z, ids, w), (z,), zeros),
                             (lambda z, o, a, f: policy.forward_backward(z, ids, o, a, f, w), (z, old, adv, ref), zeros),
                             (lambda z, f: pref.forward_backward(z, ids, starts, f, w), (z, ref), zeros + [10])):
        want, got = call(*args), call(*bad(args))
        assert _same(got, want) and bool((got[-1][gone] == 0).all()) and bool(torch.isfinite(got[-1].float()).all())
        if len(got[0]) == rows:
            assert bool((got[0][gone] == 0).all())
    w[out_by_id] = 0.0
    want = distill.forward_backward(z, at, tl, weights=w)
    z2, tl2 = bad((z, tl))
    got = distill.forward_backward(z2, at, tl2, weights=w)
    assert _same(got, want) and bool((got[1][zeros] == 0).all()) and bool((got[0][zeros] == 0).all())
    # none counts
    none = torch.zeros(rows, device=DEV)
    nan = torch.full_like(z, float("nan"))
    for out in (token.forward_backward(nan, ids, none), policy.forward_backward(nan, ids, old, adv, ref, none),
                distill.forward_backward(nan, at, tl, weights=none)):
        assert all(bool((t == 0).all()) for t in out)
    loss, rewards, dz = pref.forward_backward(nan, ids, starts, ref, none)
    assert bool((dz == 0).all()) and bool((rewards == 0).all()) and abs(float(loss[0]) - np.log(2)) <= U
    # a gradient of 0 by the log probability
    g = torch.zeros(rows, device=DEV)
    assert bool((token.logp_backward(nan, ids, g, g) == 0).all())


@pytest.mark.parametrize("dtype,vocab", [("bf16", 9), ("f32", 9), ("bf16", 1001), ("f32", 5000), ("bf16", 140001), ("f32", 70001)])
def test_infinities_and_nan(dtype, vocab):
    """Columns of -inf are as if they were not there; a row of nothing else, one with NaN or +inf, and one whose id is nowhere are NaN,
    and only they."""
    rows, ops = 8, _ops()
    rng = np.random.default_rng(3)
    t, z = logits(rng, rows, vocab, dtype)
    gone = rng.random((rows, vocab)) < 0.4
    ids = rng.integers(0, vocab, rows)
    gone[np.arange(rows), ids] = False
    z[gone] = -np.inf
    t = torch.from_numpy(z).to(TORCH[dtype]).to(DEV)
    op = ops.DeviceTokenLoss(vocab, dtype, scale=0.75)
    want, _, want_d = O.token_loss(z, ids, None, 0.75)
    loss, d = op.forward_backward(t, dev(ids, torch.int64))
    close(loss, want, delta(vocab) + U * np.abs(want), "loss")
    finite = np.where(gone, -1e30, z)
    close(d, want_d, gradient_bound(want_d, finite, 0.75, np.ones(rows), ids, dtype), "dlogits")
    assert bool((d[dev(gone, torch.bool)] == 0).all())

    sick = t.clone()
    sick[1], sick[2, vocab // 2], sick[3, vocab - 1] = float("-inf"), float("nan"), float("inf")
    where = dev(ids, torch.int64)
    where[4], where[5] = vocab, -7
    one = torch.ones(rows, device=DEV)
    for got in (op.forward_backward(sick, where), ops.DevicePolicyLoss(vocab, dtype).forward_backward(sick, where, -2 * one, one)):
        rowwise = [got[0], got[-1].float().sum(1)]
        for x in rowwise:
            assert torch.isnan(x).tolist() == [i in (1, 2, 3, 4, 5) for i in range(rows)], x
    alone = op.forward_backward(t[6:], where[6:])
    both = op.forward_backward(sick, where)
    assert torch.equal(both[1][6:], alone[1]) and torch.equal(both[0][6:], alone[0])
    logp, lse = op.logp(sick, where)
    assert float(lse[1]) == -np.inf and torch.isnan(logp).tolist() == [i in (1, 2, 3, 4, 5) for i in range(rows)]
    d = op.logp_backward(t, where, lse.nan_to_num(0, 0, 0), torch.ones(rows, device=DEV))
    assert torch.isnan(d.float()).any(1).tolist() == [i in (4, 5) for i in range(rows)]
    # a token of probability 0
    t[0, 0], where[0] = float("-inf"), 0
    loss, d = op.forward_backward(t, where)
    assert float(loss[0]) == np.inf and bool(torch.isfinite(d[0].float()).all()) and float(d[0, 0]) == -0.75


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distillation_of_masked_columns(dtype):
    vocab = 50
    rng = np.random.default_rng(4)
    t, z = logits(rng, 4, vocab, dtype)
    at = np.stack([rng.permutation(vocab)[:6] for _ in range(4)])
    tl = rng.standard_normal((4, 6)).astype(np.float32)
    lse = f32([O.softmax(x)[1] + 0.5 for x in tl])
    z[1, 30:] = -np.inf
    z[1, at[1]] = 1.0
    others = np.ones(vocab, bool)
    others[at[2]] = False
    z[2, others] = -np.inf                                          # what is left over has no column: no rest
    z[3, at[3, 0]] = -np.inf                                        # the teacher says what the student excludes
    zd = torch.from_numpy(z).to(TORCH[dtype])
    op = _ops().DeviceDistillation(vocab, dtype)
    for given in (None, lse):
        loss, d = op.forward_backward(zd.to(DEV), dev(at, torch.int64), dev(tl), top_lse=dev(given))
        with np.errstate(divide="ignore"):
            want, want_d = O.distill_loss(zd.double().numpy(), at, tl, given)
        assert float(loss[3]) == np.inf == want[3]
        close(loss[:3], want[:3], 4 * (delta(vocab) + 4 * U) + 2 * U * np.abs(want[:3]), "loss")
        close(d, want_d, HALF_STEP[dtype] * np.abs(want_d) + 60 * U + 4 * delta(vocab), "dlogits")


def test_ratios_out_of_range():
    """exp(logp - old) overflows: clipped where the advantage is positive, infinite where it is negative, nothing where it is 0"""
    vocab = 100
    z = torch.randn(4, vocab, device=DEV)
    ids = torch.randint(0, vocab, (4,), device=DEV)
    adv = dev([1.0, -1.0, 0.0, 1.0])
    old = dev([-500.0, -500.0, -500.0, 500.0])
    loss, logp, d = _ops().DevicePolicyLoss(vocab, "f32").forward_backward(z, ids, old, adv)
    assert abs(float(loss[0]) + 1.2) < 1e-6 and float(loss[1]) == np.inf and float(loss[2]) == 0 and float(loss[3]) == 0
    assert bool((d[0] == 0).all()) and bool((d[2:] == 0).all())


@pytest.mark.parametrize("name", NAMES)
def test_gradient_against_differences(name):
    """Along g the losses' sum changes by 2 e |g|^2 between z + e g and z - e g.  In fp32 the sum of 11 losses near 10 is off by about 11 x 10 x
    2^-24 x a few; e makes the change 0.02, and terms of the third order are (0.02 / 10)^2 of it.  Together 1 %.  (The policy's ratios
    are near 1 for that: with losses of 1000, e g would be less than the last bit of z.)"""
    rows, vocab = 11, 300
    call = _calls(vocab, "f32", rows, seed=9)[name]
    z = 2 * torch.randn(rows, vocab, device=DEV)
    if name == "logp":
        ops = _ops().DeviceTokenLoss(vocab, "f32")
        ids, g = torch.randint(0, vocab, (rows,), device=DEV), torch.randn(rows, device=DEV)
        lse = ops.logp(z, ids)[1]
        d = ops.logp_backward(z, ids, lse, g)
        value = lambda z: float((ops.logp(z, ids)[0].double() * g).sum())
    else:
        if name == "policy":
            ids, r = torch.randint(0, vocab, (rows,), device=DEV), lambda: torch.randn(rows, device=DEV)
            lp = _ops().DeviceTokenLoss(vocab, "f32").logp(z, ids)[0]
            op, old, adv, ref = _ops().DevicePolicyLoss(vocab, "f32", kl=0.1), lp + 0.03 * r(), r(), lp + 0.3 * r()
            call = lambda z: op.forward_backward(z, ids, old, adv, ref)
        d = call(z)[-1]
        value = lambda z: float(call(z)[0].double().sum())
    square = float((d.double() ** 2).sum())
    e = 0.01 / square
    assert abs(value(z + e * d) - value(z - e * d) - 0.02) <= 0.01 * 0.02


def test_shards_add_up():
    rows, vocab, n = 37, 999, 3
    rng = np.random.default_rng(8)
    t, z = logits(rng, rows, vocab, "f32")
    ids = rng.integers(0, vocab, rows)
    ids[3] = -1
    part = vocab // n
    shards = [_ops().DeviceTokenLoss(part, "f32", first_id=i * part, whole_vocab=vocab) for i in range(n)]
    zs = [t[:, i * part:(i + 1) * part].to(DEV) for i in range(n)]
    idt = dev(ids, torch.int64)
    logp, lse = zip(*(op.logp(x, idt) for op, x in zip(shards, zs)))
    whole = torch.logsumexp(torch.stack(lse).double(), 0).float()
    logp = (torch.stack(logp).double() + torch.stack(lse).double()).sum(0) - whole.double()
    on = ids >= 0
    want, _ = O.logp(z, ids)
    close(logp.cpu()[on], want[on], 4 * delta(vocab) + 16 * U * 12, "logp")
    g = f32(rng.standard_normal(rows))
    d = torch.cat([op.logp_backward(x, idt, whole, dev(g)) for op, x in zip(shards, zs)], 1)
    lse64 = whole.double().cpu().numpy()
    want_d = O.logp_bwd(z, ids, lse64, g)
    close(d, want_d, gradient_bound(want_d, z, 1.0, g, ids, "f32", lse=lse64), "dlogits")


def test_beyond_32_bits():
    """The last rows of more than 2^32 bytes and 2^31 elements are as those rows alone"""
    rows, vocab = 34000, 65536
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    z[-3:] = 3 * torch.randn(3, vocab, device=DEV)
    ids = torch.randint(0, vocab, (rows,), device=DEV)
    w = torch.zeros(rows, device=DEV)
    w[-3:] = 1.0
    op = _ops().DeviceTokenLoss(vocab)
    want = op.forward_backward(z[-3:], ids[-3:])
    logp, lse = op.logp(z[-3:], ids[-3:])
    g = torch.zeros(rows, device=DEV)
    g[-3:] = 1.0
    every = torch.zeros(rows, device=DEV)
    every[-3:] = lse
    out = torch.full_like(z, 5.0)
    d = op.logp_backward(z, ids, every, g, out=out)
    assert torch.equal(d[-3:], op.logp_backward(z[-3:], ids[-3:], lse, g[-3:])) and not bool(d[:-3].any())
    loss, d = op.forward_backward(z, ids, w, out=z)
    assert torch.equal(d[-3:], want[1]) and torch.equal(loss[-3:], want[0]) and not bool(d[:-3].any())


@pytest.mark.parametrize("name", NAMES)
def test_no_rows(name):
    got = _calls(40, "bf16", 3)
    ops, empty = _ops(), torch.empty(0, 40, dtype=torch.bfloat16, device=DEV)
    ids, f = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    starts = dev([0, 0, 0], torch.int32)
    if name == "token":
        assert ops.DeviceTokenLoss(40).forward_backward(empty, ids)[1].shape == (0, 40)
    if name == "logp":
        assert ops.DeviceTokenLoss(40).logp_backward(empty, ids, f, f).shape == (0, 40)
    if name == "policy":
        assert ops.DevicePolicyLoss(40).forward_backward(empty, ids, f, f)[0].shape == (0,)
    if name == "preference":
        loss, rewards, d = ops.DevicePreferenceLoss(40).forward_backward(empty, ids, starts)
        assert abs(float(loss[0]) - np.log(2)) <= U and bool((rewards == 0).all()) and d.shape == (0, 40)
        z = torch.randn(3, 40, device=DEV).bfloat16()              # rows, but no pair
        loss, rewards, d = ops.DevicePreferenceLoss(40).forward_backward(z, ids.new_zeros(3), dev([1], torch.int32))
        assert loss.shape == (0,) and bool((d == 0).all())
    if name in ("distill", "rest"):
        assert ops.DeviceDistillation(40).forward_backward(empty, ids.view(0, 1).expand(0, 4).contiguous(), f.view(0, 1).expand(0, 4).contiguous())[
            0].shape == (0,)


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """Replays with other logits between eager calls of the same object, on the same stream"""
    rows, vocab = 19, 3001
    call = _calls(vocab, "bf16", rows)[name]
    z = (2 * torch.randn(rows, vocab, device=DEV)).bfloat16()
    want = call(z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call(z)
    for i in range(4):
        z.copy_((2 * torch.randn(rows, vocab, device=DEV)).bfloat16())
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            eager = call(z)
        torch.cuda.synchronize()
        assert _same(out, eager) and not _same(out[:1], want[:1])


def test_threads_on_one_stream():
    """The preference loss has three launches and scratch memory between them"""
    import threading
    op = _ops().DevicePreferenceLoss(500)
    jobs = []
    for rows in (6, 300, 1000):
        z = torch.randn(rows, 500, device=DEV).bfloat16()
        ids, starts = torch.randint(0, 500, (rows,), device=DEV), dev([0, rows // 2, rows], torch.int32)
        jobs.append(lambda z=z, i=ids, s=starts: op.forward_backward(z, i, s))
    want = [j() for j in jobs]
    torch.cuda.synchronize()
    meet, wrong = threading.Barrier(len(jobs)), []

    def work(job, expect):
        meet.wait(30)
        got = [job() for _ in range(30)]
        torch.cuda.synchronize()
        wrong.extend(i for i, g in enumerate(got) if not _same(g, expect))
    threads = [threading.Thread(target=work, args=a) for a in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not any(t.is_alive() for t in threads) and not wrong
