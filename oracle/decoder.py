"""Definition, in NumPy fp64 and without any tiling, of the operators around a decoder block: embedding lookup, per-head RMS norm
with the position rotation, and cross attention, each with its gradient."""
import numpy as np


# ---- embedding ------------------------------------------------------------------------------------

def embed_fwd(table, ids, scale=1.0, first_row=0):
    """y[t] = scale * table[ids[t] - first_row], or zeros where that is no row of the table"""
    y = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(np.asarray(ids, dtype=np.int64)):
        if first_row <= i < first_row + table.shape[0]:
            y[t] = scale * table[i - first_row].astype(np.float64)
    return y


def embed_bwd(rows, ids, dy, scale=1.0, first_row=0, pad_id=-1):
    g = np.zeros((rows, dy.shape[1]))
    for t, i in enumerate(np.asarray(ids, dtype=np.int64)):
        if first_row <= i < first_row + rows and i != pad_id:
            g[i - first_row] += scale * dy[t].astype(np.float64)
    return g


# ---- head norm and rotation -----------------------------------------------------------------------

def rotate(n, cos, sin, pos, rot, pairs, back=False):
    """n [batch, tokens, heads, columns]; pos [batch, tokens]; columns (i, i + rot / 2), or (2 i, 2 i + 1), by angle i"""
    y = n.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        c, s = cos[pos, i].astype(np.float64)[..., None], sin[pos, i].astype(np.float64)[..., None]
        if back:
            s = -s
        y[..., a] = n[..., a] * c - n[..., b] * s
        y[..., b] = n[..., b] * c + n[..., a] * s
    return y


def head_norm_fwd(x, gain, cos, sin, pos, rot, pairs, eps):
    x = x.astype(np.float64)
    u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(u * (1.0 if gain is None else gain.astype(np.float64)), cos, sin, pos, rot, pairs)


def head_norm_bwd(x, dy, gain, cos, sin, pos, rot, pairs, eps):
    """(dx, dgain)"""
    x = x.astype(np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x * r
    dn = rotate(dy.astype(np.float64), cos, sin, pos, rot, pairs, back=True)
    du = dn * (1.0 if gain is None else gain.astype(np.float64))
    return r * (du - u * (du * u).mean(-1, keepdims=True)), (dn * u).sum((0, 1, 2))


# ---- cross attention ------------------------------------------------------------------------------

def keys_that_count(batch, k_len, key_lens=None, key_mask=None):
    on = np.ones((batch, k_len), bool)
    if key_lens is not None:
        on &= np.arange(k_len)[None] < np.asarray(key_lens)[:, None]
    if key_mask is not None:
        on &= np.asarray(key_mask, bool)
    return on


def cross_fwd(q, k, v, scale, key_lens=None, key_mask=None):
    """q [batch, queries, heads, dh], k, v [batch, keys, key heads, dh] -> (o, lse [batch, heads, queries]).  Keys that do not
    count are left out altogether; a query without a key, or whose scores are all -inf, gives zeros and -inf."""
    b, n, hq, dh = q.shape
    on, g = keys_that_count(b, k.shape[1], key_lens, key_mask), hq // k.shape[2]
    o, lse = np.zeros(q.shape), np.full((b, hq, n), -np.inf)
    for i in range(b):
        for h in range(hq):
            kk, vv = k[i, on[i], h // g].astype(np.float64), v[i, on[i], h // g].astype(np.float64)
            if len(kk) == 0:
                continue
            with np.errstate(invalid="ignore"):
                s = scale * (q[i, :, h].astype(np.float64) @ kk.T)
                top = s.max(-1, keepdims=True)
                p = np.exp(s - np.where(top == -np.inf, 0.0, top))
                total = p.sum(-1, keepdims=True)
                some = total[:, 0] != 0
                o[i, some, h] = (p[some] / total[some]) @ vv
                lse[i, h, some] = (top + np.log(np.where(total == 0, 1.0, total)))[some, 0]
    return o, lse


def cross_bwd(q, k, v, do, scale, key_lens=None, key_mask=None):
    """(dq, dk, dv)"""
    b, n, hq, dh = q.shape
    on, g = keys_that_count(b, k.shape[1], key_lens, key_mask), hq // k.shape[2]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for i in range(b):
        at = np.flatnonzero(on[i])
        if len(at) == 0:
            continue
        for h in range(hq):
            qq, dd = q[i, :, h].astype(np.float64), do[i, :, h].astype(np.float64)
            kk, vv = k[i, at, h // g].astype(np.float64), v[i, at, h // g].astype(np.float64)
            s = scale * (qq @ kk.T)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            dp = dd @ vv.T
            ds = p * (dp - (p * dp).sum(-1, keepdims=True))
            dq[i, :, h] = scale * (ds @ kk)
            dk[i, at, h // g] += scale * (ds.T @ qq)
            dv[i, at, h // g] += p.T @ dd
    return dq, dk, dv
