"""What the operators around the block refuse, and with which status, before anything reaches a GPU; sizes of their scratch."""
import os

import pytest

from paper_2504_03662_amd import binding as gx

P = 1 << 20                                # an address that is never followed: every call here ends before a launch


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(gx.LIB_PATH):
        from paper_2504_03662_amd.build import build
        build(verbose=False)
    return gx.lib()


def _embed(**kw):
    d = dict(tokens=10, hidden=64, rows=100, dtype=gx.GX_BF16, id_bytes=8, flags=0, first_row=0, pad_id=-1, scale=1.0)
    d.update(kw)
    return gx.EmbedCfg(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), 2), (dict(tokens=(1 << 24) + 1), 2), (dict(rows=0), 2), (dict(rows=(1 << 24) + 1), 2), (dict(hidden=0), 2),
    (dict(hidden=65544), 2), (dict(hidden=68), 3), (dict(dtype=gx.GX_F32, hidden=66), 3), (dict(dtype=2), 4), (dict(id_bytes=2), 4),
    (dict(flags=1), 6), (dict(first_row=-1), 2), (dict(pad_id=-2), 2)])
def test_embedding_refuses(kw, status):
    c = _embed(**kw)
    assert gx.embed_fwd(c, P, P, P, check=False) == status
    assert gx.embed_bwd(c, P, P, P, P, check=False) == status
    assert gx.embed_workspace_bytes(c) == 0


def test_embedding_pointers():
    c = _embed()
    for k in range(3):
        args = [P] * 3
        args[k] = None
        assert gx.embed_fwd(c, *args, check=False) == 1
        args[k] = P + 4
        assert gx.embed_fwd(c, *args, check=False) == 5
    for k in range(4):
        args = [P] * 4
        args[k] = None
        assert gx.embed_bwd(c, *args, check=False) == 1
        args[k] = P + 4
        assert gx.embed_bwd(c, *args, check=False) == 5
    assert gx.embed_fwd(_embed(tokens=0), None, None, None, check=False) == gx.GX_OK
    with pytest.raises(gx.GxError, match="gx_embed_fwd"):
        gx.embed_fwd(c, P, None, P)


def test_embedding_scratch_grows_with_tokens():
    sizes = [gx.embed_workspace_bytes(_embed(tokens=t)) for t in (1, 17, 1000, 5000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    # two copies of (row, token), and at least the partial sums of the pieces
    assert sizes[3] >= 4 * 4 * 5000


def _norm(**kw):
    d = dict(batch=2, q_len=3, k_len=4, q_heads=8, k_heads=2, head_dim=64, rot_dim=64, max_pos=10, dtype=gx.GX_BF16, flags=0,
             eps=1e-6)
    d.update(kw)
    return gx.HeadsNormCfg(*d.values())


class _View:
    """Something with an address, strides and a shape, as a tensor has them"""

    def __init__(self, strides=(4096, 1024, 64, 1), address=P, shape=(2, 3, 8, 64)):
        self.strides, self.address, self.shape = strides, address, shape

    def stride(self):
        return self.strides

    def data_ptr(self):
        return self.address


def _norm_in(q=None, k=None, **kw):
    d = dict(q_gain=P, k_gain=P, q_pos=P, k_pos=P, cos_table=P, sin_table=P)
    d.update(kw)
    return gx.heads_norm_in(q or _View(), k or _View(), *d.values())


def _both(c, i, out=None):
    o = out or _View()
    return {gx.heads_norm_fwd(c, i, o, o, check=False),
            gx.heads_norm_bwd(c, i, _View(), _View(), o, o, P, P, P, check=False)}


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 2), (dict(q_len=-1), 2), (dict(k_heads=-2), 2), (dict(head_dim=0), 2), (dict(head_dim=264), 2),
    (dict(head_dim=60, rot_dim=0), 3), (dict(rot_dim=24), 3), (dict(rot_dim=80), 2), (dict(rot_dim=-16), 2), (dict(max_pos=-1), 2),
    (dict(dtype=5), 4), (dict(flags=2), 6), (dict(eps=-1.0), 2), (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2)])
def test_head_norm_refuses(kw, status):
    assert _both(_norm(**kw), _norm_in()) == {status}
    assert gx.heads_norm_workspace_bytes(_norm(**kw)) == 0


def test_head_norm_pointers_and_strides():
    c = _norm()
    assert _both(c, _norm_in(q=_View(address=0))) == {1}
    assert _both(c, _norm_in(cos_table=None)) == {1}
    assert _both(c, _norm_in(sin_table=P + 8)) == {5}
    assert _both(c, _norm_in(q_gain=P + 2)) == {5}
    assert _both(c, _norm_in(k_pos=P + 2)) == {5}
    assert _both(c, _norm_in(k=_View(address=P + 8))) == {5}
    assert _both(c, _norm_in(q=_View(strides=(4096, 1023, 64, 1)))) == {5}
    assert _both(c, _norm_in(q=_View(strides=(4096, -1024, 64, 1)))) == {2}
    # outputs may not repeat; inputs may; strides of an extent of 1 do not matter
    assert _both(c, _norm_in(), _View(strides=(4096, 1024, 0, 1))) == {2}
    reached = 7                                                    # no gfx950 here: the last check before a launch
    import torch
    if not torch.cuda.is_available():
        assert _both(c, _norm_in(q=_View(strides=(0, 1024, 0, 1)))) == {reached}
        one = _norm(batch=1, q_len=1, k_len=1)
        assert _both(one, _norm_in(q=_View(strides=(3, -7, 64, 1)))) == {reached}
        assert gx.heads_norm_fwd(_norm(k_len=0), _norm_in(k=_View(address=0)), _View(), None, check=False) == reached
    assert gx.heads_norm_bwd(c, _norm_in(), _View(), _View(), _View(), _View(), P, P, None, check=False) == 1
    assert gx.heads_norm_bwd(c, _norm_in(q_gain=None), _View(), _View(), _View(), _View(), P, None, P, check=False) == 1
    assert gx.heads_norm_bwd(c, _norm_in(), _View(), _View(), _View(), _View(), P + 4, P, P, check=False) == 5
    with pytest.raises(ValueError, match="contiguous columns"):
        gx.heads(_View(strides=(4096, 1024, 64, 2)))


def _cross(**kw):
    d = dict(batch=2, q_len=3, k_len=3, q_heads=8, k_heads=8, head_dim=64, dtype=gx.GX_BF16, flags=0, scale=0.125)
    d.update(kw)
    return gx.CrossCfg(*d.values())


def _cross_in(q=None, k=None, v=None, lens=None, mask=None):
    return gx.cross_in(q or _View(), k or _View(), v or _View(), lens, mask)


def _cross_both(c, i, out=None):
    o = out or _View()
    return {gx.cross_fwd(c, i, o, P, P, check=False), gx.cross_bwd(c, i, _View(), P, _View(), o, o, o, P, check=False)}


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 2), (dict(q_len=-1), 2), (dict(k_len=-1), 2), (dict(k_len=(1 << 22) + 1), 2), (dict(q_heads=0), 2),
    (dict(k_heads=3), 3), (dict(q_heads=4), 3), (dict(head_dim=96), 2), (dict(head_dim=256), 2),
    (dict(head_dim=62, dtype=gx.GX_F32), 3), (dict(head_dim=132, dtype=gx.GX_F32), 2), (dict(dtype=3), 4), (dict(flags=1), 6),
    (dict(scale=0.0), 2), (dict(scale=-1.0), 2), (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2),
    (dict(q_len=1 << 28), 2), (dict(batch=1 << 22, k_len=4096), 2)])
def test_cross_attention_refuses(kw, status):
    assert _cross_both(_cross(**kw), _cross_in()) == {status}
    assert gx.cross_workspace_bytes(_cross(**kw), False) == gx.cross_workspace_bytes(_cross(**kw), True) == 0


def test_cross_attention_pointers_and_strides():
    c = _cross()
    assert _cross_both(c, _cross_in(k=_View(address=0))) == {1}
    assert _cross_both(c, _cross_in(v=_View(address=P + 8))) == {5}
    assert _cross_both(c, _cross_in(lens=P + 2)) == {5}
    assert _cross_both(c, _cross_in(q=_View(strides=(4096, 1022, 64, 1)))) == {5}
    assert _cross_both(c, _cross_in(k=_View(strides=(4096, 32, 64, 1)))) == {2}          # tokens of keys overlap
    assert _cross_both(c, _cross_in(v=_View(strides=(4096, 1 << 23, 64, 1)))) == {2}
    assert _cross_both(c, _cross_in(), _View(strides=(0, 1024, 64, 1))) == {2}             # outputs that repeat
    far = _View(strides=(1 << 34, 1024, 1 << 31, 1))
    assert gx.cross_fwd(_cross(k_heads=1), _cross_in(q=far), _View(), P, P, check=False) == 2
    good = _View()
    assert gx.cross_bwd(c, _cross_in(), good, None, good, good, good, good, P, check=False) == 1
    assert gx.cross_bwd(c, _cross_in(), good, P, good, good, good, good, None, check=False) == 1
    assert gx.cross_bwd(c, _cross_in(), good, P, _View(address=0), good, good, good, P, check=False) == 1
    assert gx.cross_fwd(c, _cross_in(), good, P + 2, P, check=False) == 5
    import torch
    if not torch.cuda.is_available():                              # the last check before a launch
        assert _cross_both(c, _cross_in(k=_View(strides=(0, 1024, 0, 1)))) == {7}
        assert _cross_both(_cross(k_len=0), _cross_in(k=_View(address=0), v=_View(address=0))) == {7}
        assert gx.cross_fwd(c, _cross_in(), good, None, None, check=False) == 7


def test_cross_attention_scratch():
    # one query against a long cache is split and needs room for the parts: sums, reference and total of a row each
    one = _cross(batch=1, q_len=1, k_len=8192, q_heads=8, k_heads=8)
    n = gx.cross_workspace_bytes(one, False)
    assert n > 0 and n % (8 * (64 + 2) * 4) == 0
    # work for the whole chip is not
    assert gx.cross_workspace_bytes(_cross(batch=8, q_len=2048, k_len=2048, q_heads=16, k_heads=16), False) == 0
    for dtype in (gx.GX_BF16, gx.GX_F32):
        for q, k in ((0, 0), (0, 100), (100, 0)):
            assert gx.cross_workspace_bytes(_cross(q_len=q, k_len=k, dtype=dtype), False) >= 0
        # D and lse of every row at least
        assert gx.cross_workspace_bytes(_cross(q_len=500, k_len=64, dtype=dtype), True) >= 2 * 4 * 2 * 8 * 500
