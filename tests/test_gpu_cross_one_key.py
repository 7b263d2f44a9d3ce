"""Rows that see one key or a few.  One: P is 1, o is that key's value to the bit, and dP = D, so that dQ and dK are exactly zero, in both types, whole
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


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("m,lens", [(2, None), (3, None), (13, None), (700, (2, 3, 2)), (20000, (3, 2, 2))])
def test_few_keys(dh, m, lens):
    """bf16, a few keys to a row, also where the others are cut off and where the keys are split: dQ and dK have two roundings, of dS and
    of the result, each off by at most 2^-8 / sqrt(3) of what is rounded in the mean square; P's own 2^-10 adds a 30th to one
    of them.  D must not add the rounding of o."""
    rng = np.random.default_rng([20250403, 831, m, dh])
    b, n, hq, hk = 3, 150 if m < 20000 else 5, 8, 2
    q, k, v, do = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16().to(DEV)
                   for s in ((b, n, hq, dh), (b, m, hk, dh), (b, m, hk, dh), (b, n, hq, dh)))
    op = DeviceCrossAttention(dh)
    key_lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = op.forward(q, k, v, key_lens)
    dq, dk, dv = op.backward(q, k, v, o, lse, do, key_lens)
    off = [0.0, 0.0]
    size = [0.0, 0.0]
    for i in range(b):
        c = m if lens is None else lens[i]
        x = [t[i, :c] if t.shape[1] == m else t[i] for t in (q, k, v, do)]
        qq, kk, vv, dd = (t.double().cpu().numpy().transpose(1, 0, 2) for t in x)
        kk, vv = (np.repeat(t, hq // hk, 0) for t in (kk, vv))
        s = qq @ kk.transpose(0, 2, 1) * dh ** -0.5
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        dp = dd @ vv.transpose(0, 2, 1)
        ds = p * (dp - (p * dp).sum(-1, keepdims=True)) * dh ** -0.5
        want = (ds @ kk).transpose(1, 0, 2), (ds.transpose(0, 2, 1) @ qq).reshape(hk, hq // hk, c, dh).sum(1).transpose(1, 0, 2)
        for j, (got, w) in enumerate(zip((dq[i], dk[i, :c]), want)):
            off[j] += ((got.double().cpu().numpy() - w) ** 2).sum()
            size[j] += (w ** 2).sum()
    for j in range(2):
        assert (off[j] / size[j]) ** 0.5 <= (2.0 + 1 / 30) ** 0.5 * 2.0 ** -8 / 3 ** 0.5, (j, (off[j] / size[j]) ** 0.5)
