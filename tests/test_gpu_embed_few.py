"""The table's gradient for few tokens (one launch) and at the size where the sorted form takes over, to the bounds of the other
embedding tests: n terms, off by at most (n + 2) 2^-24 of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

from test_gpu_embed import DEV, _check_gradient, _inputs
from paper_2504_03662_amd.decoder_ops import DeviceEmbedding

pytestmark = pytest.mark.gpu


# hidden: one lane, a part of a block of columns, several blocks and a part; rows: one, more than a workgroup's, many; all tokens
# different to all alike (16 and 17 of a row: the ends of the two ways to add)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,hidden,rows,hot", [(1, 8, 70001, 0), (16, 1032, 1, 0), (17, 1032, 1, 0), (64, 520, 3, 0.5), (511, 264, 5000, 0.1),
                                                    (512, 2056, 129, 1.0), (512, 8, 2100000, 0.3), (513, 72, 40, 0.5)])
def test_few_tokens(tokens, hidden, rows, hot, dtype):
    table, ids, dy = _inputs(tokens, hidden, rows, rows, dtype, 40 + tokens, hot)
    op, i64 = DeviceEmbedding(rows, hidden, dtype, scale=1.5), torch.from_numpy(ids).to(DEV)
    out = torch.full((rows, hidden), float("nan"), device=DEV)
    g = op.backward(i64, dy, out=out)
    if rows * hidden <= 1 << 21:
        _check_gradient(g, rows, ids, dy, 1.5, 0, -1)
    else:                                                          # the rows with a token, and nothing anywhere else
        rest = torch.ones(rows, dtype=torch.bool, device=DEV)
        rest[i64] = False
        assert not g[rest].any()
        some, where = np.unique(ids, return_inverse=True)
        _check_gradient(g[torch.from_numpy(some).to(DEV)], len(some), where, dy, 1.5, 0, -1)
    assert torch.equal(op.backward(i64.int(), dy), g)
    base = torch.randn(rows, hidden, device=DEV)
    added = op.backward(i64, dy, out=base.clone(), accumulate=True)
    if rows * hidden <= 1 << 21:
        _check_gradient(added, rows, ids, dy, 1.5, 0, -1, base.double().cpu().numpy())
    assert torch.equal(op.backward(i64, dy, out=base.clone(), accumulate=True), added)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_tokens_of_a_shard_with_padding(dtype):
    rows, vocab, first, hidden, tokens = 333, 1000, 400, 40, 300
    table, ids, dy = _inputs(tokens, hidden, rows, vocab, dtype, 6, 0.3)
    ids[:7] = [first - 1, first, first + rows - 1, first + rows, -1, 2 ** 40, -(2 ** 62)]
    i64 = torch.from_numpy(ids).to(DEV)
    dy[torch.from_numpy(np.flatnonzero(ids == vocab // 2)).to(DEV)[0]] = float("inf")
    for pad in (vocab // 2, first - 1):
        g = DeviceEmbedding(rows, hidden, dtype, first_row=first, pad_id=pad).backward(i64, dy)
        if pad == vocab // 2:
            _check_gradient(g, rows, ids, torch.nan_to_num(dy, posinf=0.0), 1.0, first, pad)
        else:                                                      # the infinity stays in its row
            assert (g[vocab // 2 - first] == float("inf")).all()
            assert g[torch.arange(rows, device=DEV) != vocab // 2 - first].isfinite().all()
