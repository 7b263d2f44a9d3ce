"""Rows that see one key: P is 1, o is that key's value to the bit, and dP = D, so that dQ and dK are exactly zero, in both types, whole
or split, wherever the key stands."""
import numpy as np
import pytest
import torch

from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 20), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n,m,hq,hk", [(170, 1, 4, 1), (1, 1, 2, 2), (33, 700, 4, 2), (600, 40, 2, 2), (1, 5000, 8, 1)])
def test_one_key(dtype, dh, n, m, hq, hk):
    rng = np.random.default_rng([20250403, 830, n, m])
    b, t = 3, torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, do = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(t).to(DEV)
                   for s in ((b, n, hq, dh), (b, m, hk, dh), (b, m, hk, dh), (b, n, hq, dh)))
    at = rng.integers(0, m, b)
    mask = torch.zeros(b, m, dtype=torch.bool)
    mask[torch.arange(b), torch.from_numpy(at)] = True
    mask = mask.to(DEV) if m > 1 else None
    op = DeviceCrossAttention(dh, dtype)
    o, lse = op.forward(q, k, v, key_mask=mask)
    dq, dk, dv = op.backward(q, k, v, o, lse, do, key_mask=mask)
    for i in range(b):
        want = v[i, at[i]].repeat_interleave(hq // hk, 0)[None].expand(n, hq, dh)
        assert torch.equal(o[i], want)
        # P is off by what its exponent is rounded by: 2^-20 or so of 1, then the sum over rows and the output's rounding
        total = do[i].double().view(n, hk, hq // hk, dh)
        err = (dv[i, at[i]].double() - total.sum((0, 2))).abs()
        bound = 2.0 ** -8 * total.abs().sum((0, 2)) if dtype == "bf16" else 2.0 ** -19 * total.abs().sum((0, 2))
        assert bool((err <= bound + 2.0 ** -126).all())
    assert float(dq.abs().max()) == 0.0 and float(dk.abs().max()) == 0.0
