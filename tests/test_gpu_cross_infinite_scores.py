"""Cross attention of queries whose scores that count are all -inf: as if no key counted, o is 0, lse -inf, and there is no gradient to
the queries, keys or values."""
import pytest
import torch

from test_gpu_cross import DEV, _inputs
from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 20), ("f32", 128)]


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("n,m", [(1, 1), (1, 5000), (33, 40), (64, 64), (70, 700), (300, 130)])
@pytest.mark.parametrize("masked", [False, True])
def test_queries_whose_scores_are_all_minus_infinity(dtype, dh, n, m, masked):
    """The first of two key heads holds only -inf; the second one's results are those that it has without the first"""
    q, k, v, do = _inputs(2, n, m, 4, 2, dh, dtype, seed=10)
    q = q.abs() + 0.125
    mask = None
    if masked:
        mask = torch.rand(2, m, device=DEV) < 0.7
        mask[:, 0] = True
    op = DeviceCrossAttention(dh, dtype)
    o, lse = op.forward(q, k, v, key_mask=mask)
    want = (o, lse.transpose(1, 2)) + op.backward(q, k, v, o, lse, do, key_mask=mask)
    k[:, :, 0] = float("-inf")
    o, lse = op.forward(q, k, v, key_mask=mask)
    got = (o, lse.transpose(1, 2)) + op.backward(q, k, v, o, lse, do, key_mask=mask)
    for name, g, w in zip(("o", "lse", "dq", "dk", "dv"), got, want):
        first, heads = g.shape[2] // 2, g[:, :, :g.shape[2] // 2]
        assert (heads == float("-inf")).all() if name == "lse" else not heads.any(), name
        assert torch.equal(g[:, :, first:], w[:, :, first:]), name
