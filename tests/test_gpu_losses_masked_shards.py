"""Log probabilities over shards of which some hold nothing but -inf in a row: a shard of padding, or of columns that a mask excludes"""
import numpy as np
import pytest
import torch

from loss_cases import DEV, TORCH, U, close, delta, dev, f32, gradient_bound, logits
from oracle import losses as O

pytestmark = pytest.mark.gpu


def _shard(vocab, dtype, i, n, **kw):
    from paper_2504_03662_amd.loss_ops import DeviceTokenLoss
    return DeviceTokenLoss(vocab // n, dtype, first_id=i * (vocab // n), whole_vocab=vocab, **kw)


def _whole(logp, lse):
    """The documented way"""
    lse, logp = torch.stack(lse).double(), torch.stack(logp).double()
    whole = torch.logsumexp(lse, 0)
    return (logp + lse.masked_fill(lse == float("-inf"), 0.0)).sum(0) - whole, whole


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [24, 3003, 24000, 200001])
def test_shards_of_nothing_add_up(vocab, dtype):
    rows, n = 12, 3
    part = vocab // n
    rng = np.random.default_rng(vocab)
    t, z = logits(rng, rows, vocab, dtype)
    ids = np.concatenate([rng.integers(0, part, 4), rng.integers(part, 2 * part, 4), rng.integers(2 * part, vocab, 4)])
    z[0:2, part:2 * part] = -np.inf                                 # another shard than the token's
    z[2, part:] = -np.inf                                           # both others
    z[4, :part] = -np.inf
    z[5, part:2 * part] = -np.inf                                   # the token's own: no such token
    z[6, :2 * part] = -np.inf                                       # and one more
    z[9, :] = -np.inf                                               # no token at all
    ids[10] = -1
    ids[11] = vocab                                                 # of no shard
    z[11, :part] = -np.inf
    t = torch.from_numpy(z).to(TORCH[dtype])
    idt = dev(ids, torch.int64)
    shards, zs = [_shard(vocab, dtype, i, n) for i in range(n)], [t[:, i * part:(i + 1) * part].contiguous().to(DEV) for i in range(n)]
    logp, lse = zip(*(op.logp(x, idt) for op, x in zip(shards, zs)))
    for i in range(n):
        want, want_lse = O.logp(z[:, i * part:(i + 1) * part], np.where(ids == vocab, -1, ids), first=i * part)
        sane = [r for r in range(rows) if r != 11]                  # (the oracle knows no such id)
        none = np.flatnonzero(np.isneginf(want_lse))
        assert np.isneginf(lse[i].cpu().numpy()[sane]).nonzero()[0].tolist() == none.tolist() and 9 in none
        assert logp[i].cpu().numpy()[none].tolist() == [-np.inf if i * part <= ids[r] < (i + 1) * part else 0.0 for r in none]
        some = [r for r in sane if r not in none]
        close(lse[i].cpu()[some], want_lse[some], delta(part) + U * (1 + np.abs(want_lse[some])), "a shard's lse")
        close(logp[i].cpu()[some], want[some], delta(part) + U * (1 + np.abs(want_lse[some]) + np.abs(want[some])), "a shard's logp")
        assert torch.isnan(logp[i][11])
    got, whole = _whole(logp, lse)
    assert got[[5, 6]].tolist() == [-np.inf] * 2 and bool(torch.isnan(got[[9, 11]]).all()) and float(whole[9]) == -np.inf
    sane = [0, 1, 2, 3, 4, 7, 8]
    want, want_lse = O.logp(z, np.where(ids == vocab, -1, ids))
    close(got.cpu()[sane], want[sane], 4 * delta(vocab) + 16 * U * 12, "logp")
    # the gradient by it
    whole = whole.float()
    g = f32(rng.standard_normal(rows))
    g[9] = g[11] = 0.0
    d = torch.cat([op.logp_backward(x, idt, whole, dev(g)) for op, x in zip(shards, zs)], 1)
    lse64 = whole.double().cpu().numpy()
    want_d = O.logp_bwd(z, np.where(ids == vocab, -1, ids), lse64, g)
    rest = [r for r in range(rows) if r != 9]
    assert not d[9].any()
    close(d[rest], want_d[rest], gradient_bound(want_d[rest], np.where(np.isneginf(z), -1e30, z)[rest], 1.0, g[rest],
                                               np.where(ids == vocab, -1, ids)[rest], dtype, lse=lse64[rest]), "dlogits")


def test_a_shard_of_the_lowest_number():
    """lse rounds to -inf there at a scale of 2"""
    t = torch.zeros(3, 20, device=DEV)
    t[:, 10:] = torch.finfo(torch.float32).min
    ids = dev([3, 13, 3], torch.int64)
    logp, lse = zip(*(_shard(20, "f32", i, 2, scale=2.0).logp(t[:, 10 * i:10 * i + 10].contiguous(), ids) for i in range(2)))
    assert lse[1].tolist() == [-np.inf] * 3 and logp[1].tolist() == [0.0, -np.inf, 0.0]
    got, _ = _whole(logp, lse)
    assert got[1] == -np.inf and float((got[[0, 2]] + np.log(10)).abs().max()) <= 4 * (delta(10) + 4 * U)


def test_the_whole_vocabulary_of_nothing_is_still_nan():
    from paper_2504_03662_amd.loss_ops import DeviceTokenLoss
    t = torch.full((2, 30), float("-inf"), device=DEV)
    logp, lse = DeviceTokenLoss(30, "f32").logp(t, dev([1, 29], torch.int64))
    assert bool(torch.isnan(logp).all()) and lse.tolist() == [-np.inf] * 2
