"""Embedding lookup and the table's gradient on the GPU against the 64-bit definition, to bounds that follow from the arithmetic:
the lookup is one fp32 product rounded once to the storage type (bit-exact), and an element of the gradient is a sum of
n fp32 terms times the scale, off by at most (n + 2) 2^-24 of the sum of the terms' magnitudes, whatever the order."""
import numpy as np
import pytest
import torch

from oracle import decoder as D
from paper_2504_03662_amd.decoder_ops import DeviceEmbedding
from paper_2504_03662_amd.runtime import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(tokens, hidden, rows, vocab, dtype, seed, hot=0.0):
    rng = np.random.default_rng([20250403, 800, seed])
    table = torch.from_numpy(rng.standard_normal((rows, hidden)).astype(np.float32)).to(TYPES[dtype]).to(DEV)
    dy = torch.from_numpy(rng.standard_normal((tokens, hidden)).astype(np.float32)).to(TYPES[dtype]).to(DEV)
    ids = rng.integers(0, vocab, tokens)
    ids[rng.random(tokens) < hot] = vocab // 2                     # one token makes up a part of the text
    return table, ids, dy


def _check_gradient(got, rows, ids, dy, scale, first, pad, base=None):
    got, d = got.double().cpu().numpy(), to_host(dy)
    want = D.embed_bwd(rows, ids, d, scale, first, pad)
    size = D.embed_bwd(rows, ids, np.abs(d), abs(scale), first, pad)
    n = D.embed_bwd(rows, ids, np.ones_like(d), 1.0, first, pad)
    if base is not None:
        want, size, n = want + base, size + np.abs(base), n + 1
    bad = np.abs(got - want) > (n + 2) * 2.0 ** -24 * size
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


# one piece, the ends of a piece (16) and of a block of the sort (4096), several of them; narrow and wide rows; one row of the
# vocabulary, and enough for two and three passes of the sort
@pytest.mark.parametrize("tokens,hidden,rows,hot", [
    (1, 8, 1, 0), (2, 64, 5, 0), (15, 24, 3, 0), (16, 8, 100, 0), (17, 72, 1, 0), (33, 256, 1000, 0.5), (257, 264, 511, 0),
    (1000, 2056, 512, 0.3), (4095, 16, 70000, 0), (4096, 64, 40, 0), (4097, 8, 300000, 0.9), (9001, 136, 513, 0.25),
    (20000, 16, 2, 0.5)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lookup_and_gradient(tokens, hidden, rows, hot, dtype):
    table, ids, dy = _inputs(tokens, hidden, rows, rows, dtype, tokens, hot)
    op = DeviceEmbedding(rows, hidden, dtype, scale=1.5)
    i64 = torch.from_numpy(ids).to(DEV)
    y = op.forward(table, i64)
    assert torch.equal(y, (table[i64].float() * 1.5).to(TYPES[dtype]))
    g = op.backward(i64, dy)
    _check_gradient(g, rows, ids, dy, 1.5, 0, -1)
    assert torch.equal(op.backward(i64.int(), dy), g)              # the other id type, the same bits


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shard_and_padding(dtype):
    rows, vocab, first, hidden, tokens = 333, 1000, 400, 40, 2500
    table, ids, dy = _inputs(tokens, hidden, rows, vocab, dtype, 5, 0.2)
    ids[:4] = [first - 1, first, first + rows - 1, first + rows]
    ids[4:7] = [-1, 2 ** 40, -(2 ** 62)]                           # ids of no row at all
    i64 = torch.from_numpy(ids).to(DEV)
    for pad in (-1, vocab // 2, first, 3):
        op = DeviceEmbedding(rows, hidden, dtype, first_row=first, pad_id=pad)
        assert np.array_equal(to_host(op.forward(table, i64)), D.embed_fwd(to_host(table), ids, 1.0, first))
        _check_gradient(op.backward(i64, dy), rows, ids, dy, 1.0, first, pad)


def test_no_token_of_this_shard():
    op = DeviceEmbedding(10, 16, "f32", first_row=100)
    ids, dy = torch.arange(50, device=DEV), torch.ones(50, 16, device=DEV)
    assert not op.forward(torch.ones(10, 16, device=DEV), ids).any()
    out = torch.full((10, 16), 7.0, device=DEV)
    assert not op.backward(ids, dy, out=out).any()
    out.fill_(7.0)
    assert (op.backward(ids, dy, out=out, accumulate=True) == 7.0).all()


def test_no_tokens():
    op = DeviceEmbedding(10, 16, "bf16")
    ids, dy = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, 16, dtype=torch.bfloat16, device=DEV)
    assert op.forward(torch.ones(10, 16, dtype=torch.bfloat16, device=DEV), ids).shape == (0, 16)
    out = torch.full((10, 16), 7.0, device=DEV)
    assert (op.backward(ids, dy, out=out, accumulate=True) == 7.0).all()
    assert not op.backward(ids, dy, out=out).any()


def test_accumulates_and_repeats_bit_for_bit():
    rows, hidden, tokens = 200, 128, 6000
    table, ids, dy = _inputs(tokens, hidden, rows, rows, "bf16", 9, 0.4)
    op, i64 = DeviceEmbedding(rows, hidden, "bf16", scale=0.5), torch.from_numpy(ids).to(DEV)
    base = torch.randn(rows, hidden, device=DEV)
    got = [op.backward(i64, dy, out=base.clone(), accumulate=True) for _ in range(3)]
    _check_gradient(got[0], rows, ids, dy, 0.5, 0, -1, base.double().cpu().numpy())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    shape = (3, 2000)
    assert torch.equal(op.backward(i64.view(shape), dy.view(*shape, hidden)), op.backward(i64, dy))
    assert op.forward(table, i64.view(shape)).shape == (*shape, hidden)


def test_a_value_that_is_not_finite_stays_in_its_row():
    ids = torch.tensor([1, 2, 2, 3, 2, 4] * 20, device=DEV)
    dy = torch.ones(120, 8, device=DEV)
    dy[ids == 3] = float("nan")
    dy[0] = float("inf")
    g = DeviceEmbedding(6, 8, "f32").backward(ids, dy)
    assert g[3].isnan().all() and (g[1] == float("inf")).all() and (g[2] == 60).all() and (g[4] == 20).all()
    assert not g[0].any() and not g[5].any()


def test_replays_from_a_captured_graph_and_on_another_stream():
    rows, hidden, tokens = 5000, 256, 3000
    table, ids, dy = _inputs(tokens, hidden, rows, rows, "bf16", 11, 0.1)
    op, i64 = DeviceEmbedding(rows, hidden, "bf16"), torch.from_numpy(ids).to(DEV)
    want = op.backward(i64, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = op.backward(i64, dy)
        out = torch.empty_like(want)
        op.backward(i64, dy, out=out)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        op.backward(i64, dy, out=out)
    for k in range(3):
        dy.mul_(-1.0)
        want = op.backward(i64, dy)                                # eager, on the scratch of this stream
        out.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
