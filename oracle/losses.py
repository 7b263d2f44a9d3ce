"""Definition, in NumPy fp64 and row by row, of the losses of logits with their gradients: log probabilities and cross entropy, the
clipped policy loss, the preference loss of pairs and distillation from a teacher's top logits."""
import numpy as np

IGNORE = -1


def softmax(a):
    """(p, lse)"""
    with np.errstate(invalid="ignore"):
        top = a.max()
        e = np.exp(a - top)
        return e / e.sum(), top + np.log(e.sum())


def _row(z, scale):
    return scale * z.astype(np.float64)


def logp(z, ids, scale=1.0, ignore=IGNORE, first=0):
    """(logp, lse) by row; a token of another shard has -lse, and in a shard of nothing but -inf lse is not taken from anything"""
    out = np.zeros((2, len(ids)))
    for t, i in enumerate(ids):
        if i != ignore:
            a = _row(z[t], scale)
            lse = softmax(a)[1] if a.max() != -np.inf else -np.inf
            out[:, t] = (a[i - first] if first <= i < first + len(a) else 0.0) - (lse if lse != -np.inf else 0.0), lse
    return out[0], out[1]


def logp_bwd(z, ids, lse, dlogp, scale=1.0, ignore=IGNORE, first=0):
    d = np.zeros(z.shape)
    for t, i in enumerate(ids):
        g = scale * np.float64(dlogp[t])
        if i != ignore and g != 0:
            d[t] = -g * np.exp(_row(z[t], scale) - np.float64(lse[t]))
            if first <= i < first + z.shape[1]:
                d[t, i - first] += g
    return d


def _whole(z, ids, weights, scale, ignore, loss_of):
    """Losses and gradients of rows that count: loss_of(t, logp) -> (loss, its derivative by logp), without the weight"""
    loss, d, lp = np.zeros(len(ids)), np.zeros(z.shape), np.zeros(len(ids))
    for t, i in enumerate(ids):
        w = 1.0 if weights is None else np.float64(weights[t])
        if i == ignore or w == 0:
            continue
        a = _row(z[t], scale)
        p, lse = softmax(a)
        lp[t] = a[i] - lse
        l, g = loss_of(t, lp[t])
        loss[t] = w * l
        d[t] = -w * g * scale * p
        # 1 - p without the difference
        d[t, i] = w * g * scale * np.delete(p, i).sum()
    return loss, lp, d


def token_loss(z, ids, weights=None, scale=1.0, ignore=IGNORE):
    """(loss, logp, dlogits)"""
    return _whole(z, ids, weights, scale, ignore, lambda t, lp: (-lp, -1.0))


def policy_loss(z, ids, old, adv, ref=None, weights=None, low=0.2, high=0.2, kl=0.0, scale=1.0, ignore=IGNORE):
    """(loss, logp, dlogits)"""
    def of(t, lp):
        r, a = np.exp(lp - np.float64(old[t])), np.float64(adv[t])
        l = g = 0.0
        if a != 0:
            cut = min(max(r, 1.0 - low), 1.0 + high)
            l = -min(r * a, cut * a)
            g = -r * a if r * a <= cut * a else 0.0
        if kl:
            d = np.float64(ref[t]) - lp
            l += kl * (np.expm1(d) - d)
            g -= kl * np.expm1(d)
        return l, g
    return _whole(z, ids, weights, scale, ignore, of)


def pairs_loss(lp, starts, ref=None, weights=None, pair_weights=None, beta=0.1, margin=0.0, smoothing=0.0):
    """(loss, rewards, dlogp)"""
    n, pairs = len(lp), len(starts) // 2
    w = np.ones(n) if weights is None else np.asarray(weights, np.float64)
    gain = np.zeros(n)
    on = w != 0
    gain[on] = w[on] * (np.asarray(lp, np.float64)[on] - (0.0 if ref is None else np.asarray(ref, np.float64)[on]))
    at = np.clip(starts, 0, n)
    loss, rewards, d = np.zeros(pairs), np.zeros(2 * pairs), np.zeros(n)
    for j in range(2 * pairs):
        rewards[j] = beta * gain[at[j]:at[j + 1]].sum()
    for i in range(pairs):
        pw = 1.0 if pair_weights is None else np.float64(pair_weights[i])
        if pw == 0:
            continue
        x = rewards[2 * i] - rewards[2 * i + 1] - margin
        # a part of factor 0 is none, also where x is infinite
        loss[i] = pw * sum(f * np.logaddexp(0, y) for f, y in ((1 - smoothing, -x), (smoothing, x)) if f)
        slope = pw * beta * (smoothing - np.exp(-np.logaddexp(0, x)))
        d[at[2 * i]:at[2 * i + 1]] = slope
        d[at[2 * i + 1]:at[2 * i + 2]] = -slope
    return loss, rewards, d * w


def preference_loss(z, ids, starts, ref=None, weights=None, pair_weights=None, beta=0.1, margin=0.0, smoothing=0.0, scale=1.0,
                    ignore=IGNORE):
    """(loss, rewards, dlogits)"""
    w = np.ones(len(ids)) if weights is None else np.array(weights, np.float64)
    w[np.asarray(ids) == ignore] = 0.0
    lp = token_loss(z, ids, w, scale, ignore)[1]
    loss, rewards, g = pairs_loss(lp, starts, ref, w, pair_weights, beta, margin, smoothing)
    return loss, rewards, token_loss(z, ids, -g, scale, ignore)[2]


def distill_loss(z, top_ids, top_logits, top_lse=None, weights=None, scale=1.0):
    """(loss, dlogits)"""
    n, vocab = z.shape
    loss, d = np.zeros(n), np.zeros(z.shape)
    for t in range(n):
        w = 1.0 if weights is None else np.float64(weights[t])
        on = (top_ids[t] >= 0) & (top_ids[t] < vocab)
        if w == 0 or not on.any():
            continue
        at = top_ids[t][on]
        logq = scale * top_logits[t][on].astype(np.float64)
        logq = logq - (softmax(logq)[1] if top_lse is None else np.float64(top_lse[t]))
        a = _row(z[t], scale)
        p, lse = softmax(a)
        q = np.exp(logq)
        others = np.ones(vocab, bool)
        others[at] = False
        for lq, qi, col in zip(logq, q, at):
            if qi != 0:
                loss[t] += qi * (lq - (a[col] - lse))
        r = 0.0
        if top_lse is not None and others.any() and a[others].max() > -np.inf:
            r = max(0.0, 1.0 - q.sum())
        if r > 0:
            p_others, lse_others = softmax(a[others])
            loss[t] += r * (np.log(r) - (lse_others - lse))
            d[t, others] -= r * p_others
        d[t] += (q.sum() + r) * p
        np.subtract.at(d[t], at, q)
        loss[t] *= w
        d[t] *= w * scale
    return loss, d
