"""Queries or keys without a token (or without a head): the sum over no tokens is zero, so that a gain's gradient that is asked for is
zeros, or unchanged where it is added to."""
import pytest
import torch

from paper_2504_03662_amd import binding as gx
from paper_2504_03662_amd.decoder_ops import DeviceHeadNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [8, 64, 200])
@pytest.mark.parametrize("q_shape,k_shape", [((2, 0, 4), (2, 5, 2)), ((2, 5, 4), (2, 0, 2)), ((2, 5, 0), (2, 5, 2)), ((1, 0, 4), (1, 0, 2)),
                                             ((3, 7, 0), (3, 0, 1))])
def test_gain_gradient_of_an_empty_side(dtype, dh, q_shape, k_shape):
    t = TYPES[dtype]
    q, dyq = (torch.randn(*q_shape, dh, device=DEV).to(t) for _ in range(2))
    k, dyk = (torch.randn(*k_shape, dh, device=DEV).to(t) for _ in range(2))
    gq, gk = torch.ones(dh, dtype=t, device=DEV), torch.full((dh,), 0.5, dtype=t, device=DEV)
    op = DeviceHeadNorm(dh, 0, dtype)
    alone = {"q": op.backward(q, None, dyq, None, gq)[2] if q.numel() else torch.zeros(dh, device=DEV),
             "k": op.backward(None, k, None, dyk, None, gk)[3] if k.numel() else torch.zeros(dh, device=DEV)}
    nan = lambda: torch.full((dh,), float("nan"), device=DEV)
    # written whole, into the caller's tensors and into new ones (which likely take the memory of the two that are dropped here)
    outs = nan(), nan()
    dq, dk, dgq, dgk = op.backward(q, k, dyq, dyk, gq, gk, dgain_q=outs[0], dgain_k=outs[1])
    assert dgq is outs[0] and dgk is outs[1] and dq.shape == q.shape and dk.shape == k.shape
    assert torch.equal(dgq, alone["q"]) and torch.equal(dgk, alone["k"])
    del dgq, dgk, outs
    again = op.backward(q, k, dyq, dyk, gq, gk)[2:]
    assert torch.equal(again[0], alone["q"]) and torch.equal(again[1], alone["k"])
    # one empty side on its own
    for side, x in (("q", q), ("k", k)):
        if x.numel() == 0:
            out = nan()
            if side == "q":
                op.backward(q, None, dyq, None, gq, dgain_q=out)
            else:
                op.backward(None, k, None, dyk, None, gk, dgain_k=out)
            assert not out.any()
    # added to: nothing
    base = torch.randn(dh, device=DEV), torch.randn(dh, device=DEV)
    outs = base[0].clone(), base[1].clone()
    op.backward(q, k, dyq, dyk, gq, gk, dgain_q=outs[0], dgain_k=outs[1], accumulate=True)
    for x, b, o in ((q, base[0], outs[0]), (k, base[1], outs[1])):
        assert torch.equal(o, b) == (x.numel() == 0)


def test_an_empty_sides_gradient_is_checked_too():
    x, gain = torch.ones(1, 0, 2, 64, device=DEV), torch.ones(64, device=DEV)
    with pytest.raises(gx.GxError) as e:
        DeviceHeadNorm(64, 0, "f32").backward(x, None, x, None, gain, dgain_q=torch.ones(65, device=DEV)[1:])
    assert e.value.status == 5                                     # 16 bytes
