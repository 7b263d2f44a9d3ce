"""Tokens whose position the tables do not have: NaN in every column, whether or not it is turned, forward and backward, and in no
other token; the gains' gradients, sums over all tokens, are NaN.  Without a rotation positions do not matter."""
import pytest
import torch

from paper_2504_03662_amd.decoder_ops import DeviceHeadNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dh,rot,heads", [(48, 16, 3), (128, 64, 2), (256, 16, 1), (64, 64, 5), (24, 16, 70)])
def test_a_position_outside_the_tables(dtype, pairs, dh, rot, heads):
    t, n = TYPES[dtype], 9
    x, dy = (torch.randn(2, n, heads, dh, device=DEV).to(t) for _ in range(2))
    gain = torch.randn(dh, device=DEV).to(t)
    angle = torch.rand(6, rot // 2, device=DEV)
    cos, sin = angle.cos(), angle.sin()
    there = torch.randint(0, 6, (2, n), device=DEV, dtype=torch.int32)
    pos = there.clone()
    out = [(0, 1, -1), (0, 4, 6), (0, 5, 7), (1, 0, 2 ** 31 - 1), (1, 8, -2 ** 31)]
    for b, i, p in out:
        pos[b, i] = p
    bad = torch.zeros(2, n, dtype=torch.bool, device=DEV)
    bad[[o[0] for o in out], [o[1] for o in out]] = True
    op = DeviceHeadNorm(dh, rot, dtype, pairs=pairs)
    for side in ("q", "k"):
        both = lambda p: dict(cos=cos, sin=sin, q_pos=p) if side == "q" else dict(cos=cos, sin=sin, k_pos=p)
        fwd = lambda p: op.forward(x, None, gain, **both(p))[0] if side == "q" else op.forward(None, x, None, gain, **both(p))[1]
        bwd = lambda p: (op.backward(x, None, dy, None, gain, **both(p))[::2] if side == "q"
                         else op.backward(None, x, None, dy, None, gain, **both(p))[1::2])
        y, want = fwd(pos), fwd(there)
        assert y[bad].isnan().all() and torch.equal(y[~bad], want[~bad]) and want.isfinite().all()
        (dx, dgain), (want, sums) = bwd(pos), bwd(there)
        assert dx[bad].isnan().all() and torch.equal(dx[~bad], want[~bad]) and want.isfinite().all()
        assert dgain.isnan().all() and sums.isfinite().all()


def test_positions_do_not_matter_without_a_rotation():
    x = torch.randn(1, 3, 2, 64, device=DEV)
    pos = torch.tensor([[-1, 5, 2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    op = DeviceHeadNorm(64, 0, "f32")
    assert torch.equal(op.forward(x, None, q_pos=pos)[0], op.forward(x)[0])
    assert torch.equal(op.backward(x, None, x, None, q_pos=pos)[0], op.backward(x, None, x, None)[0])
