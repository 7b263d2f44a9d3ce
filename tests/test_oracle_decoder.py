"""Pins of oracle/decoder.py: closed forms, identities and central differences of every gradient."""
import numpy as np
import pytest

from oracle import decoder as D

RNG = np.random.default_rng(20250403)


def _differences(f, x, h=1e-5):
    """gradient of the scalar f(x) by central differences"""
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_embedding_is_a_product_with_one_hot_rows():
    table, ids = RNG.standard_normal((7, 5)), np.array([3, 9, 4, 3, 2, 10, -1, 8])
    one_hot = (ids[:, None] == np.arange(3, 10)[None]).astype(float)             # rows 3 .. 9 of a vocabulary
    assert np.allclose(D.embed_fwd(table, ids, 2.0, 3), 2.0 * one_hot @ table, atol=1e-15)
    dy = RNG.standard_normal((8, 5))
    assert np.allclose(D.embed_bwd(7, ids, dy, 2.0, 3), 2.0 * one_hot.T @ dy, atol=1e-15)
    g = D.embed_bwd(7, ids, dy, 2.0, 3, pad_id=3)
    assert not g[0].any() and np.array_equal(g[1:], D.embed_bwd(7, ids, dy, 2.0, 3)[1:])


def test_shards_of_the_vocabulary_add_up():
    table, ids, dy = RNG.standard_normal((12, 4)), RNG.integers(0, 12, 30), RNG.standard_normal((30, 4))
    whole = D.embed_fwd(table, ids)
    assert np.array_equal(whole, sum(D.embed_fwd(table[r:r + 4], ids, 1.0, r) for r in (0, 4, 8)))
    assert np.allclose(D.embed_bwd(12, ids, dy), np.concatenate([D.embed_bwd(4, ids, dy, 1.0, r) for r in (0, 4, 8)]))


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_keeps_lengths_and_depends_on_differences_of_positions(pairs):
    rot, pos = 8, np.array([[5, 11, 0]])
    angle = np.arange(40)[:, None] * np.array([1.0, 0.3, 0.1, 0.02])
    cos, sin = np.cos(angle), np.sin(angle)
    x, y = RNG.standard_normal((1, 3, 2, 12)), RNG.standard_normal((1, 3, 2, 12))
    turn = lambda z, p: D.rotate(z, cos, sin, p, rot, pairs)
    assert np.allclose((turn(x, pos) ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose((turn(x, pos) * turn(y, pos + 3)).sum(-1), (turn(x, pos + 20) * turn(y, pos + 23)).sum(-1))
    assert np.allclose(D.rotate(turn(x, pos), cos, sin, pos, rot, pairs, back=True), x)
    assert np.array_equal(turn(x, pos)[:, 2], x[:, 2])                           # position 0
    assert np.array_equal(turn(x, pos)[..., rot:], x[..., rot:])
    i, j = (2, 3) if pairs else (1, 5)                                           # angle 1 turns these two
    e = np.zeros((1, 1, 1, 12))
    e[..., i] = 1.0
    z = turn(e, np.array([[5]]))[0, 0, 0]
    assert np.isclose(z[i], np.cos(1.5)) and np.isclose(z[j], np.sin(1.5))


@pytest.mark.parametrize("pairs", [False, True])
def test_head_norm_gradients_by_differences(pairs):
    rot, pos, eps = 4, np.array([[1, 7], [3, 0]]), 1e-3
    angle = np.arange(9)[:, None] * np.array([1.0, 0.2])
    a = (np.cos(angle), np.sin(angle), pos, rot, pairs, eps)
    x, gain, dy = RNG.standard_normal((2, 2, 2, 6)), 1 + 0.2 * RNG.standard_normal(6), RNG.standard_normal((2, 2, 2, 6))
    dx, dg = D.head_norm_bwd(x, dy, gain, *a)
    assert np.allclose(dx, _differences(lambda z: (dy * D.head_norm_fwd(z, gain, *a)).sum(), x), atol=1e-7)
    assert np.allclose(dg, _differences(lambda z: (dy * D.head_norm_fwd(x, z, *a)).sum(), gain), atol=1e-7)
    y = D.head_norm_fwd(x, None, *a)
    assert np.allclose((y ** 2).mean(-1), (x ** 2).mean(-1) / ((x ** 2).mean(-1) + eps))


def _attention_inputs(b=2, n=3, m=5, hq=4, hk=2, dh=3):
    r = RNG.standard_normal
    return r((b, n, hq, dh)), r((b, m, hk, dh)), r((b, m, hk, dh)), r((b, n, hq, dh))


def test_cross_attention_by_hand():
    # two keys with scores 0 and ln 3: weights 1/4 and 3/4
    q, k = np.array([[[[1.0, 0.0]]]]), np.array([[[[0.0, 1.0]], [[2 * np.log(3.0), 0.0]]]])
    v = np.array([[[[4.0, 0.0]], [[0.0, 8.0]]]])
    o, lse = D.cross_fwd(q, k, v, 0.5)
    assert np.allclose(o[0, 0, 0], [1.0, 6.0]) and np.isclose(lse[0, 0, 0], np.log(4.0))
    o, lse = D.cross_fwd(q, k, v, 0.5, key_lens=[1])
    assert np.allclose(o[0, 0, 0], [4.0, 0.0]) and lse[0, 0, 0] == 0.0
    o, lse = D.cross_fwd(q, k, v, 0.5, key_mask=[[False, False]])
    assert not o.any() and lse[0, 0, 0] == -np.inf


def test_cross_attention_against_torch():
    import torch
    q, k, v, do = _attention_inputs()
    mask = np.array([[1, 0, 1, 1, 1], [1, 1, 1, 0, 0]], bool)
    t = [torch.from_numpy(x).transpose(1, 2).requires_grad_() for x in (q, np.repeat(k, 2, 2), np.repeat(v, 2, 2))]
    o = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=torch.from_numpy(mask)[:, None, None], scale=0.7)
    assert np.allclose(D.cross_fwd(q, k, v, 0.7, key_mask=mask)[0], o.detach().transpose(1, 2).numpy())
    g = torch.autograd.grad(o, t, torch.from_numpy(do).transpose(1, 2))
    dq, dk, dv = D.cross_bwd(q, k, v, do, 0.7, key_mask=mask)
    group = lambda x: x.transpose(1, 2).numpy().reshape(2, 5, 2, 2, 3).sum(3)
    assert np.allclose(dq, g[0].transpose(1, 2).numpy()) and np.allclose(dk, group(g[1])) and np.allclose(dv, group(g[2]))


def test_cross_attention_gradients_by_differences():
    q, k, v, do = _attention_inputs()
    where = dict(key_lens=[4, 5], key_mask=np.array([[1, 0, 1, 1, 1], [0, 0, 0, 0, 0]], bool))
    f = lambda a, b, c: (do * D.cross_fwd(a, b, c, 0.6, **where)[0]).sum()
    dq, dk, dv = D.cross_bwd(q, k, v, do, 0.6, **where)
    assert np.allclose(dq, _differences(lambda z: f(z, k, v), q), atol=1e-8)
    assert np.allclose(dk, _differences(lambda z: f(q, z, v), k), atol=1e-8)
    assert np.allclose(dv, _differences(lambda z: f(q, k, z), v), atol=1e-8)
    assert not dq[1].any() and not dk[1].any() and not dk[0, [1, 4]].any() and not dv[0, [1, 4]].any()
