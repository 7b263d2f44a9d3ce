"""Cross attention of more samples with lengths than a wavefront sorts (64), and of exactly as many: every sample's results are those
that it has on its own, to the bounds of the other cross-attention tests."""
import numpy as np
import pytest

from test_gpu_cross import _check, _inputs, _run
from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("samples", [63, 64, 65, 130])
@pytest.mark.parametrize("n,m,hq,hk,dh,dtype", [(1, 200, 4, 2, 64, "bf16"), (40, 150, 2, 1, 128, "bf16"), (1, 90, 2, 2, 64, "f32"),
                                                (33, 70, 2, 1, 32, "f32")])
@pytest.mark.parametrize("masked", [False, True])
def test_many_samples(samples, n, m, hq, hk, dh, dtype, masked):
    case = (samples, n, m, hq, hk, dh, dtype)
    q, k, v, do = _inputs(*case, seed=11)
    rng = np.random.default_rng([20250403, 850, samples, n])
    lens = rng.integers(0, m + 1, samples)
    lens[[0, 1, samples - 1]] = 0, m, m                            # and many equal ones
    lens[5:25] = 37
    lens = [int(x) for x in lens]
    mask = (rng.random((samples, m)) < 0.8) if masked else None
    _check(q, k, v, do, dh ** -0.5, _run(DeviceCrossAttention(dh, dtype), q, k, v, do, lens, mask), dtype, lens, mask)
