"""Per-head norm and rotation on the GPU against the 64-bit definition, element by element.  With u = 2^-24: the sum of up to 256
squares, the root and the products of a column's value are off by less than 40 u of it, so that a turned pair (a, b) is off by
less than 48 u (|a| + |b|); the mean that the input gradient takes is off by less than 64 u of the mean of the
magnitudes; a gain's gradient is a sum of n such products, off by at most (n + 64) u of the sum of their magnitudes.  A bf16
output lies between the roundings of the bound's two ends."""
import numpy as np
import pytest
import torch

from oracle import decoder as D
from paper_2504_03662_amd.decoder_ops import DeviceHeadNorm
from paper_2504_03662_amd.runtime import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
EPS = 1e-6


def _tensor(rng, shape, dtype, std=1.0, mean=0.0):
    return torch.from_numpy((mean + std * rng.standard_normal(shape)).astype(np.float32)).to(TYPES[dtype]).to(DEV)


def _tables(max_pos, rot):
    half = rot // 2
    angle = np.arange(max_pos)[:, None] * 10000.0 ** (-np.arange(half) / max(half, 1))
    return [torch.from_numpy(f(angle).astype(np.float32)).to(DEV) for f in (np.cos, np.sin)]


def _near(name, got, want, bound, dtype):
    got = to_host(got).astype(np.float64)
    bound = bound + 1e-38
    if dtype == "bf16":
        # rounding is monotonic: what lies within the bound rounds to between these two
        lo, hi = (torch.from_numpy(np.float32(x)).bfloat16().double().numpy() for x in (want - bound, want + bound))
    else:
        lo, hi = want - bound, want + bound
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), (name, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


def _check(x, y, dy, dx, dgain, gain, cos, sin, pos, rot, pairs, dtype, base=None):
    x, dy, gain = to_host(x), to_host(dy), None if gain is None else to_host(gain)
    where = (to_host(cos), to_host(sin), pos, rot, pairs)
    plus = (np.abs(where[0]), -np.abs(where[1]), pos, rot, pairs)          # |a| |c| + |b| |s| in the first of a pair
    gabs = None if gain is None else np.abs(gain)

    def pair_sum(n):                                                      # |a| + |b| of a column's pair
        s = np.abs(n)
        t = s.copy()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            t[..., a] = t[..., b] = s[..., a] + s[..., b]
        return t

    r = 1.0 / np.sqrt((x.astype(np.float64) ** 2).mean(-1, keepdims=True) + EPS)
    u, g = x * r, 1.0 if gain is None else gain.astype(np.float64)
    _near("y", y, D.head_norm_fwd(x, gain, *where, EPS), 48 * U * pair_sum(u * g), dtype)
    want, wgain = D.head_norm_bwd(x, dy, gain, *where, EPS)
    dn = pair_sum(dy)
    du = dn * np.abs(g)
    mean = (du * np.abs(u)).mean(-1, keepdims=True)
    _near("dx", dx, want, 64 * U * r * (du + 2 * np.abs(u) * mean), dtype)
    if gain is not None:
        size, n = (dn * np.abs(u)).sum((0, 1, 2)), x.shape[0] * x.shape[1] * x.shape[2]
        if base is not None:
            wgain, size = wgain + base, size + np.abs(base)
        _near("dgain", dgain, wgain, (n + 64) * U * size, "f32")


SHAPES = [  # batch, q_len, k_len, q_heads, k_heads, head_dim, rot
    (1, 1, 1, 1, 1, 8, 0), (1, 1, 1, 1, 1, 16, 16), (2, 3, 1, 5, 2, 32, 32), (3, 7, 11, 8, 2, 64, 32), (2, 33, 5, 40, 8, 128, 128),
    (1, 130, 77, 3, 1, 80, 80), (2, 9, 9, 6, 3, 96, 64), (1, 5, 1029, 2, 1, 256, 256), (1, 600, 600, 9, 9, 72, 48),
    (4, 1, 1, 33, 17, 128, 112), (1, 6000, 2, 2, 1, 24, 16)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
def test_forward_and_backward(shape, dtype, pairs):
    b, sq, sk, hq, hk, dh, rot = shape
    rng = np.random.default_rng([20250403, 810, dh, sq])
    cos, sin = _tables(50, rot)
    q, k = _tensor(rng, (b, sq, hq, dh), dtype), _tensor(rng, (b, sk, hk, dh), dtype, 3.0)
    dyq, dyk = _tensor(rng, q.shape, dtype), _tensor(rng, k.shape, dtype)
    gq, gk = _tensor(rng, (dh,), dtype, 0.2, 1.0), _tensor(rng, (dh,), dtype, 0.2, 1.0)
    pq, pk = (rng.integers(0, 50, (b, n)).astype(np.int32) for n in (sq, sk))
    where = dict(cos=cos, sin=sin, q_pos=torch.from_numpy(pq).to(DEV), k_pos=torch.from_numpy(pk).to(DEV))
    op = DeviceHeadNorm(dh, rot, dtype, EPS, pairs)
    yq, yk = op.forward(q, k, gq, gk, **where)
    dq, dk, dgq, dgk = op.backward(q, k, dyq, dyk, gq, gk, **where)
    _check(q, yq, dyq, dq, dgq, gq, cos, sin, pq, rot, pairs, dtype)
    _check(k, yk, dyk, dk, dgk, gk, cos, sin, pk, rot, pairs, dtype)
    again = op.backward(q, k, dyq, dyk, gq, gk, **where)
    assert all(torch.equal(a, c) for a, c in zip(again, (dq, dk, dgq, dgk)))
    # one side alone, and without a gain
    assert torch.equal(op.forward(q, None, gq, **where)[0], yq)
    ones = torch.ones(dh, dtype=TYPES[dtype], device=DEV)
    assert torch.equal(op.forward(q, k, None, None, **where)[1], op.forward(q, k, ones, ones, **where)[1])
    assert torch.equal(op.backward(q, k, dyq, dyk, None, None, **where)[0], op.backward(q, k, dyq, dyk, ones, ones, **where)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_of_a_packed_projection_other_layouts_and_in_place(dtype):
    b, s, hq, hk, dh, rot = 2, 37, 6, 2, 64, 64
    rng = np.random.default_rng([20250403, 811])
    cos, sin = _tables(s, rot)
    qkv = _tensor(rng, (b, s, hq + 2 * hk, dh), dtype)
    q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:].clone()
    gq, gk = _tensor(rng, (dh,), dtype, 0.2, 1.0), _tensor(rng, (dh,), dtype, 0.2, 1.0)
    op = DeviceHeadNorm(dh, rot, dtype, EPS)
    yq, yk = op.forward(q.contiguous(), k.contiguous(), gq, gk, cos, sin)              # positions 0, 1, ...
    pos = torch.arange(s, device=DEV, dtype=torch.int32).repeat(b, 1)
    got = op.forward(q, k, gq, gk, cos, sin, pos, pos)
    assert torch.equal(got[0], yq) and torch.equal(got[1], yk)
    # [batch, heads, tokens, columns] in memory, and a gradient that repeats over the heads
    qt, kt = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k))
    out_q, out_k = (torch.empty(x.shape[0], x.shape[2], s, dh, dtype=x.dtype, device=DEV).transpose(1, 2) for x in (q, k))
    got = op.forward(qt, kt, gq, gk, cos, sin, q_out=out_q, k_out=out_k)
    assert got[0] is out_q and torch.equal(out_q, yq) and torch.equal(out_k, yk)
    dy = _tensor(rng, (b, s, 1, dh), dtype)
    wide_q, wide_k = dy.expand(b, s, hq, dh), dy.expand(b, s, hk, dh)
    want = op.backward(q, k, wide_q.contiguous(), wide_k.contiguous(), gq, gk, cos, sin)
    got = op.backward(qt, kt, wide_q, wide_k, gq, gk, cos, sin)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # in place, inside the packed tensor
    dq = wide_q.contiguous()
    assert torch.equal(op.backward(q, k, dq, wide_k.contiguous(), gq, gk, cos, sin, dq=dq)[0], want[0])
    op.forward(q, k, gq, gk, cos, sin, q_out=q, k_out=k)
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(qkv[:, :, hq + hk:], v)


def test_gain_gradients_accumulate():
    rng = np.random.default_rng([20250403, 812])
    q, dy = _tensor(rng, (2, 300, 4, 64), "bf16"), _tensor(rng, (2, 300, 4, 64), "bf16")
    gain, base = _tensor(rng, (64,), "bf16", 0.2, 1.0), torch.randn(64, device=DEV)
    op = DeviceHeadNorm(64, 0, "bf16", EPS)
    out = base.clone()
    dx = op.backward(q, None, dy, None, gain, dgain_q=out, accumulate=True)[0]
    y = op.forward(q, None, gain)[0]
    cos, sin = _tables(1, 0)
    _check(q, y, dy, dx, out, gain, cos, sin, np.zeros((2, 300), np.int64), 0, False, "bf16", base.double().cpu().numpy())


def test_what_is_not_finite_and_positions_outside_the_table_stay_in_their_tokens():
    rng = np.random.default_rng([20250403, 813])
    q = _tensor(rng, (1, 5, 2, 32), "f32")
    cos, sin = _tables(4, 32)
    pos = torch.tensor([[0, 4, 3, -1, 2]], dtype=torch.int32, device=DEV)
    q[0, 2, 0, 0] = float("nan")
    q[0, 4, 1, 5] = float("inf")
    y = DeviceHeadNorm(32, 32, "f32", EPS).forward(q, None, None, None, cos, sin, pos)[0]
    assert y[0, 1].isnan().all() and y[0, 3].isnan().all()                             # no such position
    assert y[0, 2, 0].isnan().all() and y[0, 4, 1].isnan().any()
    assert y[0, 0].isfinite().all() and y[0, 2, 1].isfinite().all() and y[0, 4, 0].isfinite().all()


def test_zeros_and_large_and_small_values():
    op = DeviceHeadNorm(64, 0, "f32", EPS)
    x = torch.zeros(1, 3, 1, 64, device=DEV)
    x[0, 1], x[0, 2] = 1e18, 1e-18
    y = op.forward(x)[0]
    assert not y[0, 0].any() and torch.allclose(y[0, 1], torch.ones_like(y[0, 1])) and (y[0, 2] > 0).all()
    dx = op.backward(x, None, torch.ones_like(x), None)[0]
    assert torch.allclose(dx[0, 0], torch.full_like(dx[0, 0], 1000.0)) and dx.isfinite().all()
