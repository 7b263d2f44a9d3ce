"""Who shares scratch memory of an operator: calls of one host thread on one stream, and nobody else."""
import copy
import pickle
import threading

import pytest
import torch

from paper_2504_03662_amd.decoder_ops import DeviceEmbedding, DeviceHeadNorm

OPERATORS = [lambda: DeviceEmbedding(10, 64, device="cpu"), lambda: DeviceHeadNorm(64, device="cpu")]


@pytest.fixture
def capturing(monkeypatch):
    """Whether a capture is said to be under way on the current stream"""
    state = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state[0])
    return state


@pytest.mark.parametrize("make", OPERATORS)
def test_calls_on_a_stream_share_and_the_largest_decides(make, capturing):
    op = make()
    small = op._workspace(1000, 7)
    assert small.numel() >= 1000 and op._workspace(500, 7) is small
    other = op._workspace(1000, 8)
    assert other.data_ptr() != small.data_ptr()
    large = op._workspace(5000, 7)
    assert large.numel() >= 5000 and op._workspace(1000, 7) is large and op._workspace(1000, 8) is other


@pytest.mark.parametrize("make", OPERATORS)
def test_a_captured_call_has_memory_of_its_own(make, capturing):
    """The graph goes on writing there when it is replayed, whatever calls outside of it have come to use"""
    op = make()
    eager = op._workspace(1000, 7)
    capturing[0] = True
    kept = op._workspace(1000, 7), op._workspace(200, 7)
    assert kept[0].numel() >= 1000 and len({w.data_ptr() for w in (eager, *kept)}) == 3
    capturing[0] = False
    assert op._workspace(1000, 7) is eager and op._workspace(200, 7) is eager
    fresh = make()                                                 # nor does the first call after a capture find the graph's
    capturing[0] = True
    of_graph = fresh._workspace(1000, 7)
    capturing[0] = False
    assert fresh._workspace(1000, 7).data_ptr() != of_graph.data_ptr()


@pytest.mark.parametrize("make", OPERATORS)
def test_host_threads_do_not_share(make, capturing):
    """Two threads' launches on one stream (every thread's default stream is the same) may come in any order, also one between two of
    another's call"""
    op = make()
    mine, theirs = op._workspace(1000, 7), []
    meet = threading.Barrier(3)

    def other():
        w = op._workspace(1000, 7)
        meet.wait(10)                                              # both have theirs while the other lives
        theirs.append((w, op._workspace(600, 7)))
    threads = [threading.Thread(target=other) for _ in range(2)]
    for t in threads:
        t.start()
    meet.wait(10)
    for t in threads:
        t.join(10)
    assert len({w.data_ptr() for w in (mine, theirs[0][0], theirs[1][0])}) == 3
    assert all(w is again for w, again in theirs) and op._workspace(1000, 7) is mine


@pytest.mark.parametrize("make", OPERATORS)
def test_operators_can_be_copied(make, capturing):
    op = make()
    w = op._workspace(1000, 7)
    for twin in (copy.deepcopy(op), pickle.loads(pickle.dumps(op))):
        assert twin._workspace(1000, 7).data_ptr() != w.data_ptr()
