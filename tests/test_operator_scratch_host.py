"""Who shares scratch memory of an operator: calls of one host thread on one stream, and nobody else."""
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
