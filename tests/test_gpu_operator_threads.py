"""One object, several host threads, one stream: every call of several launches gives its own results, whatever comes between its
launches."""
import threading

import pytest
import torch

from paper_2504_03662_amd import decoder_ops as ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _jobs():
    """(object, calls of different sizes on it)"""
    r = lambda *s: torch.randn(s, device=DEV).bfloat16()
    embed = ops.DeviceEmbedding(2000, 64)
    ids = [torch.randint(0, v, (n,), device=DEV) for v, n in ((2000, 900), (30, 5000), (500, 2000))]
    dys = [r(len(i), 64) for i in ids]
    yield [lambda i=i, d=d: (embed.backward(i, d),) for i, d in zip(ids, dys)]
    norm = ops.DeviceHeadNorm(64)
    xs, gain = [(r(1, n, 4, 64), r(1, n, 4, 64)) for n in (7, 900, 3000)], r(64)
    yield [lambda x=x: norm.backward(x[0], None, x[1], None, gain)[::2] for x in xs]
    cross = ops.DeviceCrossAttention(64)
    qkv = [(r(1, n, 4, 64), r(1, m, 2, 64), r(1, m, 2, 64)) for n, m in ((1, 9000), (5, 3000), (100, 700))]

    def both(q, k, v):
        o, lse = cross.forward(q, k, v)
        return (o, lse) + cross.backward(q, k, v, o, lse, q)
    yield [lambda x=x: both(*x) for x in qkv]


@pytest.mark.parametrize("job", range(3))
def test_threads_on_one_stream(job):
    calls = list(_jobs())[job]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    meet, wrong = threading.Barrier(len(calls)), []

    def work(call, expect):
        meet.wait(30)
        got = [call() for _ in range(40)]
        torch.cuda.synchronize()
        wrong.extend(i for i, g in enumerate(got) if not all(torch.equal(x, y) for x, y in zip(g, expect)))
    threads = [threading.Thread(target=work, args=a) for a in zip(calls, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not any(t.is_alive() for t in threads) and not wrong
