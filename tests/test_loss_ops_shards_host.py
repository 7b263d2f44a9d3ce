"""Shards that do not fit into their vocabulary are refused, whatever the numbers"""
import os

import pytest
import torch

from paper_2504_03662_amd import binding as gx

P = 1 << 20                                # an address that is never followed


@pytest.mark.parametrize("first,whole,fits", [(0, 100, True), (200, 300, True), (201, 300, False), (0, 99, False), (0, 1, False), (2 ** 40 - 100, 2 ** 40, True),
                                              (2 ** 40, 2 ** 40 + 100, False), (2 ** 63 - 1, 300, False), (2 ** 63 - 100, 2 ** 40, False),
                                              (-1, 300, False), (0, -1, False)])
def test_first_id(first, whole, fits):
    if not os.path.exists(gx.LIB_PATH):
        from paper_2504_03662_amd.build import build
        build(verbose=False)
    cfg = gx.LogitsCfg(10, 100, gx.GX_BF16, 8, 0, 1.0, 100, 100, first, whole, -1)
    if not fits:
        assert gx.logp_fwd(cfg, P, P, P, P, check=False) == gx.logp_bwd(cfg, P, P, P, P, P, check=False) == 2
    elif not torch.cuda.is_available():
        assert gx.logp_fwd(cfg, P, P, P, P, check=False) == gx.logp_bwd(cfg, P, P, P, P, P, check=False) == 7
