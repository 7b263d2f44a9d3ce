"""fp32 cross attention where every wavefront owns rows or keys of its own (many rows and few keys, many keys and few rows, many of
both) and where workgroups share them, to the bounds of the other cross-attention tests."""
import numpy as np
import pytest
import torch

from oracle import decoder as D
from test_gpu_cross import DEV, _check, _inputs, _run
from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [(3, 1301, 7, 8, 2, 128), (3, 1301, 45, 8, 2, 64), (3, 2100, 5, 8, 2, 20), (3, 1, 2777, 8, 8, 128),
                                  (3, 2, 3001, 8, 4, 64), (3, 3, 5003, 4, 4, 32), (3, 700, 650, 4, 2, 128), (3, 260, 33, 2, 2, 64)])
@pytest.mark.parametrize("masked", [False, True])
def test_cuts(case, masked):
    b, n, m, hq, hk, dh = case
    q, k, v, do = _inputs(*case, "f32", seed=2)
    op = DeviceCrossAttention(dh, "f32")
    lens = mask = None
    if masked:
        rng = np.random.default_rng([20250403, 822, m])
        lens, mask = [m, 0, m // 2 + 1], rng.random((b, m)) < 0.7
        on = torch.from_numpy(D.keys_that_count(b, m, lens, mask)).to(DEV)[:, :, None, None]
        k, v = (torch.where(on, x, 0.0) for x in (k, v))
        got = _run(op, q, torch.where(on, k, float("nan")), torch.where(on, v, float("inf")), do, lens, mask)
    else:
        got = _run(op, q, k, v, do)
    _check(q, k, v, do, dh ** -0.5, got, "f32", lens, mask)
    again = _run(op, q, k, v, do, lens, mask)
    assert all(torch.equal(x, y) for x, y in zip(again, got))
