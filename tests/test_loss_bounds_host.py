"""That the bounds of the tests of sure tokens and of long sums would notice sums in fp32, shown on the host"""
import numpy as np
import pytest

from loss_cases import U
from test_gpu_losses_sums import OF_SUMS
from test_gpu_losses_sure_tokens import SIZES, _sure


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_row_sum_in_fp32(size, dtype):
    rows, vocab, _, _ = size
    s = _sure(np.random.default_rng(vocab), rows, vocab, dtype, 1.0)[-1]
    off = np.abs(np.log(np.float32(1 + s).astype(float)) - np.log1p(s))
    assert np.all(off > 10 * (s * 30 * U + 2.0 ** -46 + U * s))


@pytest.mark.parametrize("rows", [1000, 2000])
def test_a_reward_in_fp32(rows):
    """A term of 1e-6 is gone next to 1024"""
    lp = -np.log1p(_sure(np.random.default_rng(rows), rows, 1001, "f32", 1.0)[-1])
    ref = np.where(np.arange(rows) % 2, -1024.0, 1024.0)
    got = np.float32(np.float32(lp) - np.float32(ref)).sum(dtype=np.float32)
    assert abs(float(got) - lp.sum()) > 10 * (np.abs(lp).sum() * 31 * U + rows * 2.0 ** -46 + OF_SUMS)
