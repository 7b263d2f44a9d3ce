"""Distillation of rows without an entry: loss 0 and a gradient of zeros, whatever the logits hold there (a padded batch's last rows)"""
import numpy as np
import pytest
import torch

from loss_cases import DEV, TORCH, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(8, 70, 5), (8, 5003, 70), (8, 20001, 5), (8, 140001, 5), (600, 20001, 70), (33000, 40, 5)])
def test_whatever_the_logits_hold(rows, vocab, top, rest, dtype):
    from paper_2504_03662_amd.loss_ops import DeviceDistillation
    rng = np.random.default_rng(top)
    z = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).to(TORCH[dtype]).to(DEV)
    at, tl = dev(rng.integers(0, vocab, (rows, top)), torch.int64), dev(rng.standard_normal((rows, top)))
    lse = dev(np.full(rows, 5.0)) if rest else None
    at[1:6] = -1
    at[2, top - 1] = vocab                                          # nor is that a column
    op = DeviceDistillation(vocab, dtype)
    want, want_d = op.forward_backward(z, at, tl, lse)
    bad = z.clone()
    bad[1], bad[2, vocab // 2], bad[3, 0], bad[4, 1::2] = float("-inf"), float("nan"), float("inf"), float("nan")
    tl[1:4] = float("nan")
    if rest:
        lse[5] = float("nan")
    inside = bad.clone()
    for z_in, out in ((bad, None), (inside, inside)):
        loss, d = op.forward_backward(z_in, at, tl, lse, out=out)
        assert not loss[1:6].any() and not d[1:6].any()
        assert torch.equal(loss, want) and torch.equal(d, want_d)
    assert torch.equal(op.forward(bad, at, tl, lse), want)
    assert bool((want[6:] != 0).all()) and bool(want_d[6:].any(1).all())
