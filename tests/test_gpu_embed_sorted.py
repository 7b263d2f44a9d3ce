"""The table's gradient by sorted tokens, which calls of more than 512 tokens take, where it can go wrong: few, one or none of the
tokens belong to the shard; they end at, before and behind the ends of a piece (16 sorted tokens); a row's tokens fill a piece, cross
one end or both; rows at the ends of a workgroup's span of the sort (64 to 2048 rows); values that are not finite.  Bounds as in
the other embedding tests: n terms, off by at most (n + 2) 2^-24 of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

from test_gpu_embed import DEV, TYPES, _check_gradient
from paper_2504_03662_amd.decoder_ops import DeviceEmbedding

pytestmark = pytest.mark.gpu
FIRST, ROWS, HIDDEN = 1000, 300, 72


def _case(own, rng, tokens=600):
    """`own` of the tokens (their rows given) among others of other shards, in random places"""
    ids = rng.integers(0, FIRST, tokens)
    ids[rng.random(tokens) < 0.5] += FIRST + ROWS
    ids[rng.permutation(tokens)[:len(own)]] = FIRST + np.asarray(own, dtype=np.int64)
    return ids


def _dy(rng, tokens, dtype, hidden=HIDDEN):
    return torch.from_numpy(rng.standard_normal((tokens, hidden)).astype(np.float32)).to(TYPES[dtype]).to(DEV)


OWN = [[], [0], [299], [0] * 15, [0] * 16, [0] * 17, [5] * 16 + [6], [5] * 15 + [6] * 2, [5] + [6] * 16, [5] * 8 + [6] * 8, [5] * 8 + [6] * 25,
       [5] * 3 + [6] * 45 + [7], list(range(33)), [63, 64] * 9, [63] * 16 + [64] * 16, [127] * 20 + [128] * 20 + [299] * 8, list(range(300))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("own", range(len(OWN)))
def test_tokens_of_the_shard(own, dtype):
    rng = np.random.default_rng([20250403, 840, own])
    ids, dy = _case(OWN[own], rng), _dy(rng, 600, dtype)
    op, i64 = DeviceEmbedding(ROWS, HIDDEN, dtype, scale=1.5, first_row=FIRST), torch.from_numpy(ids).to(DEV)
    out = torch.full((ROWS, HIDDEN), float("nan"), device=DEV)
    g = op.backward(i64, dy, out=out)
    _check_gradient(g, ROWS, ids, dy, 1.5, FIRST, -1)
    assert torch.equal(op.backward(i64.int(), dy), g)
    base = torch.randn(ROWS, HIDDEN, device=DEV)
    added = op.backward(i64, dy, out=base.clone(), accumulate=True)
    _check_gradient(added, ROWS, ids, dy, 1.5, FIRST, -1, base.double().cpu().numpy())
    untouched = np.setdiff1d(np.arange(ROWS), OWN[own])
    assert torch.equal(added[untouched], base[untouched]) and not g[untouched].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_all_padding(dtype):
    rng = np.random.default_rng([20250403, 841])
    dy = _dy(rng, 2000, dtype)
    dy[::3] = float("nan")
    ids = torch.full((2000,), FIRST + 7, device=DEV)
    op = DeviceEmbedding(ROWS, HIDDEN, dtype, first_row=FIRST, pad_id=FIRST + 7)
    assert not op.backward(ids, dy, out=torch.full((ROWS, HIDDEN), 7.0, device=DEV)).any()
    base = torch.randn(ROWS, HIDDEN, device=DEV)
    assert torch.equal(op.backward(ids, dy, out=base.clone(), accumulate=True), base)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_row(dtype):
    """Rows with one token, with a piece's and with many, tokens of other shards among them"""
    ids = torch.tensor([1, 2, 2, 3, 2, 4, 90] * 100, device=DEV)
    dy = torch.ones(700, HIDDEN, dtype=TYPES[dtype], device=DEV)
    dy[ids == 3] = float("nan")
    dy[ids == 90] = float("nan")
    dy[0, :40] = float("inf")
    g = DeviceEmbedding(80, HIDDEN, dtype).backward(ids, dy)
    assert g[3].isnan().all() and (g[1, :40] == float("inf")).all() and (g[1, 40:] == 100).all()
    assert (g[2] == 300).all() and (g[4] == 100).all() and not g[[0] + list(range(5, 80))].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,rows,hidden", [(8192, 32768, 2048), (4099, 70001, 1032)])
def test_sizes_of_training(tokens, rows, hidden, dtype):
    """Token counts by the rank law of text; the sums in 64 bits on the GPU"""
    rng = np.random.default_rng([20250403, 842, tokens])
    ids = np.minimum(np.exp(rng.random(tokens) * np.log(rows)).astype(np.int64), rows - 1) * 7919 % rows
    dy = _dy(rng, tokens, dtype, hidden)
    table = torch.randn(rows, hidden, device=DEV).to(TYPES[dtype])
    op, i64 = DeviceEmbedding(rows, hidden, dtype, scale=3.0), torch.from_numpy(ids).to(DEV)
    assert torch.equal(op.forward(table, i64), (table[i64].float() * 3.0).to(TYPES[dtype]))
    g = op.backward(i64, dy)
    some, where = np.unique(ids, return_inverse=True)
    at, where = torch.from_numpy(some).to(DEV), torch.from_numpy(where).to(DEV)
    count = torch.bincount(where, minlength=len(some)).double()[:, None]
    sums = [torch.zeros(len(some), hidden, dtype=torch.float64, device=DEV).index_add_(0, where, 3.0 * x)
            for x in (dy.double(), dy.double().abs())]
    assert bool(((g[at].double() - sums[0]).abs() <= (count + 2) * 2.0 ** -24 * sums[1]).all())
    rest = torch.ones(rows, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert not g[rest].any()
    assert torch.equal(op.backward(i64, dy), g)
