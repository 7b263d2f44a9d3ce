"""Cross attention, bf16, of more rows (queries times heads of a group) than 2^29: D and lse of a pair take more than 2 GiB, and rows
that fill up the last tile still read as zeros, which a very small lse of a real row must not replace."""
import pytest
import torch

from paper_2504_03662_amd import binding as gx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rows_beyond_the_last_of_more_than_two_to_the_29():
    n, heads, dh = 8521761, 63, 64
    assert 2 ** 29 < n * heads < 2 ** 29 + 64                      # 31 rows in the last tile of 64
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("90 GiB of memory")
    t = torch.bfloat16
    # the queries' heads are one, and so are those of o and dO: 1 x -25 x 64 / 8 = -200 is every score and lse, P is 1, o is v
    ones, zeros = (torch.full((1, n, 1, dh), x, dtype=t, device=DEV).expand(1, n, heads, dh) for x in (1.0, 0.0))
    q, o, do, v = ones, ones, zeros, torch.ones(1, 1, 1, dh, dtype=t, device=DEV)
    k = torch.full((1, 1, 1, dh), -25.0, dtype=t, device=DEV)
    lse = torch.full((1, heads, n), -200.0, device=DEV)
    dq = torch.empty(1, n, heads, dh, dtype=t, device=DEV)
    dk, dv = (torch.full((1, 1, 1, dh), float("nan"), dtype=t, device=DEV) for _ in range(2))
    cfg = gx.CrossCfg(1, n, 1, heads, 1, dh, gx.GX_BF16, 0, 0.125)
    work = torch.empty(gx.cross_workspace_bytes(cfg, True), dtype=torch.uint8, device=DEV)
    gx.cross_bwd(cfg, gx.cross_in(q, k, v), o, lse, do, dq, dk, dv, work, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert not dv.any() and not dk.any()
    assert not dq[:, ::4001].any() and not dq[:, -70:].any()
    del dq, work, lse, q, o, do, ones, zeros
    torch.cuda.empty_cache()
