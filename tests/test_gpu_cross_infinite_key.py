"""Cross attention where a key that counts holds infinities and all its scores are -inf: it weighs 0 for every query, whatever the
number of queries (tiles of 32 and 64 rows that are full, and ones that end with rows that are not there).  dQ is the formula's 0 x inf
and not looked at."""
import numpy as np
import pytest

from oracle import decoder as D
from test_gpu_cross import _bounds, _inputs, _near
from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention
from paper_2504_03662_amd.runtime import to_host

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 20), ("f32", 128)]


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("n,hq,hk", [(1, 1, 1), (3, 2, 1), (64, 2, 2), (40, 3, 1), (65, 4, 2), (700, 2, 2)])
@pytest.mark.parametrize("m", [40, 300])
def test_a_key_whose_scores_are_all_minus_infinity(dtype, dh, n, hq, hk, m):
    q, k, v, do = _inputs(1, n, m, hq, hk, dh, dtype, seed=9)
    q = q.abs() + 0.125
    k[0, 5] = float("-inf")
    op = DeviceCrossAttention(dh, dtype)
    o, lse = op.forward(q, k, v)
    dq, dk, dv = op.backward(q, k, v, o, lse, do)
    keep = np.arange(m) != 5
    assert not dk[0, 5].any() and not dv[0, 5].any()
    hosts = [to_host(x) for x in (q, k[:, keep], v[:, keep], do)]
    scale, on = dh ** -0.5, np.ones((1, m - 1), bool)
    eo, el, eq, ek, ev = _bounds(*hosts, scale, on, dtype)
    _, wk, wv = D.cross_bwd(*hosts, scale)
    _near("o", o, D.cross_fwd(*hosts[:3], scale)[0], eo, dtype)
    _near("dk", dk[:, keep], wk, ek, dtype)
    _near("dv", dv[:, keep], wv, ev, dtype)
