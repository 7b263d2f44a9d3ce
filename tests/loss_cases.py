"""Inputs and error bounds shared by the tests of the losses.

Bounds, in units of half a step of fp32, u = 2^-24, from fp32 sums over a thread's elements and fp64 from there on (the kernels go over to
fp64 sooner, after 16 bytes of logits):
  a term of a sum of exponentials, or p: its argument is rounded twice (the difference, the product), |a - max| u each, the
  exponential is off by two u, and the sum adds at most vocab / 256 + 64 terms one after another.  Weighted with p the
  arguments' part is at most about the entropy, log(vocab).  So lse is off by at most `delta`, and p by (2 |a - lse| + 8) u + delta of itself.
  what is left is the rounding of the output, u or 2^-8 of it."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": U}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda:0"
TINY = 2.0 ** -126                                  # below that numbers may become zero


def delta(vocab):
    return U * (vocab / 256 + 64 + 2 * (np.log(vocab) + 4) + 4)


def logits(rng, rows, vocab, dtype, std=2.5):
    """On the host, as numbers that the type holds exactly: (torch tensor, NumPy array)"""
    z = rng.standard_normal((rows, vocab)) * std
    z[np.arange(rows), rng.integers(0, vocab, rows)] += 10 * rng.random(rows)
    t = torch.from_numpy(z).to(TORCH[dtype])
    return t, t.double().numpy()


def placed(t, pad=0, offset=0):
    """On the GPU, as a view of columns [offset, offset + vocab) of rows that are `pad` longer; (view, the whole)"""
    whole = torch.full((t.shape[0], t.shape[1] + pad), 77.0, dtype=t.dtype, device=DEV)
    view = whole[:, offset:offset + t.shape[1]]
    view.copy_(t)
    return view, whole


def dev(x, dtype=torch.float32):
    return None if x is None else torch.as_tensor(x, dtype=dtype).to(DEV)


def f32(x):
    return np.asarray(x, np.float32)


def close(got, want, tol, name):
    got = got.detach().double().cpu().numpy() if torch.is_tensor(got) else got
    assert got.shape == np.shape(want), (name, got.shape, np.shape(want))
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], np.asarray(want)[bad][:3],
                           np.broadcast_to(tol, got.shape)[bad][:3])


def gradient_bound(want, z, scale, g, at, dtype, extra=None, lse=None):
    """dz = g scale (1_at - p): every element off by the rounding of its type, p's own error, and where the two parts cancel by theirs.
    g: bound of |g| by row; extra: g's own error by row; lse: given, and so rounded, log sums"""
    a = scale * z
    if lse is None:
        top = a.max(1, keepdims=True)
        lse = (top + np.log(np.exp(a - top).sum(1, keepdims=True)))[:, 0]
        more = 0.0
    else:
        more = 4 * U * np.abs(lse)[:, None]
    d = a - lse[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.exp(d)
        own = np.where(p == 0, 0.0, p * (2 * np.abs(d) * U + 12 * U + delta(z.shape[1]) + more))
    if at is not None:
        rows = np.flatnonzero(at >= 0)
        own[rows, at[rows]] += 12 * U + delta(z.shape[1])
    gs = np.abs(scale * np.asarray(g))[:, None]
    tol = HALF_STEP[dtype] * np.abs(want) + gs * own + TINY * (1 + gs)
    if extra is not None:
        one = p.copy()
        if at is not None:
            one[rows, at[rows]] = 1.0
        tol = tol + scale * np.asarray(extra)[:, None] * one * (1 + HALF_STEP[dtype])
    return tol
