"""A captured call of an operator keeps its scratch memory: eager calls that need more come between the replays, other tensors take
what memory there is, and neither side sees the other's numbers."""
import pytest
import torch

from paper_2504_03662_amd import decoder_ops as ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(*shape):
    return torch.randn(shape, device=DEV).bfloat16()


def _cross():
    op = ops.DeviceCrossAttention(64)
    q, k, v, do = _randn(1, 3, 8, 64), _randn(1, 700, 4, 64), _randn(1, 700, 4, 64), _randn(1, 3, 8, 64)
    q2, k2, v2 = _randn(1, 40, 8, 64), _randn(1, 20000, 4, 64), _randn(1, 20000, 4, 64)

    def call(q, k, v, do):
        o, lse = op.forward(q, k, v)
        return (o, lse) + op.backward(q, k, v, o, lse, do)
    return op, q, lambda: call(q, k, v, do), lambda: call(q2, k2, v2, q2)


def _embedding():
    op = ops.DeviceEmbedding(3000, 128)
    ids, dy = torch.randint(0, 3000, (700,), device=DEV), _randn(700, 128)
    ids2, dy2 = torch.randint(0, 40, (30000,), device=DEV), _randn(30000, 128)
    return op, dy, lambda: (op.backward(ids, dy),), lambda: (op.backward(ids2, dy2),)


def _norm():
    op = ops.DeviceHeadNorm(128)
    q, dy, gain = _randn(1, 5, 4, 128), _randn(1, 5, 4, 128), _randn(128)
    q2, dy2 = _randn(2, 3000, 8, 128), _randn(2, 3000, 8, 128)
    call = lambda q, dy: op.backward(q, None, dy, None, gain)[::2]
    return op, dy, lambda: call(q, dy), lambda: call(q2, dy2)


def _alike(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("make", [_cross, _embedding, _norm])
@pytest.mark.parametrize("first", [True, False])
def test_larger_calls_between_replays(make, first):
    """first: the capturing stream has scratch memory before the capture"""
    op, x, small, large = make()
    want, want_large = small(), large()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        if first:
            assert _alike(small(), want)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = small()
    others = []
    for i in range(4):
        with torch.cuda.stream(side):                              # eager work on the stream that was captured
            got = large() if i % 2 == 0 else small()
            # what takes the memory that a replaced block of scratch would leave
            others += [torch.full((n,), float(i), device=DEV) for n in (64, 1000, 20000, 300000) for _ in range(4)]
            x.mul_(0.5)
        side.synchronize()
        graph.replay()
        with torch.cuda.stream(side):                              # at the same time, on the other stream
            again = large()
        torch.cuda.synchronize()
        assert _alike(got, want_large if i % 2 == 0 else want) and _alike(again, want_large)
        want = small()
        assert _alike(out, want)
        assert all(bool((t == float(j // 16)).all()) for j, t in enumerate(others))


def test_graphs_of_one_object_do_not_share():
    """Two graphs, replayed at the same time on two streams"""
    op, x, small, large = _embedding()
    want = small(), large()
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for call, stream in zip((small, large), streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[0]):
            outs.append(call())
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, stream, out in zip(graphs, streams, outs):
            with torch.cuda.stream(stream):
                out[0].zero_()
                graph.replay()
        torch.cuda.synchronize()
        assert all(_alike(o, w) for o, w in zip(outs, want))
