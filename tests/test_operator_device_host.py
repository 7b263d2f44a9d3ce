"""The GPU of an operator is the current one: a stream's handle, and the default stream's above all, means nothing on another."""
import pytest
import torch

from paper_2504_03662_amd.decoder_ops import DeviceCrossAttention, DeviceEmbedding, DeviceHeadNorm

MAKE = [lambda d: DeviceEmbedding(10, 64, device=d), lambda d: DeviceHeadNorm(64, device=d), lambda d: DeviceCrossAttention(64, device=d)]


@pytest.fixture
def current(monkeypatch):
    """The number of the current GPU, of as many as you like"""
    state = [0]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state[0], raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    return state


@pytest.mark.parametrize("make", MAKE)
def test_work_goes_to_the_operators_gpu_or_nowhere(make, current):
    op = make("cuda:1")
    with pytest.raises(ValueError, match="cuda:1"):
        op._stream()
    current[0] = 1
    assert op._stream() == 101
    with pytest.raises(ValueError, match="cuda:0"):
        make("cuda:0")._stream()


@pytest.mark.parametrize("make", MAKE)
def test_a_gpu_without_a_number_is_the_current_one(make, current):
    current[0] = 3
    op = make("cuda")
    assert op.index == 3 and op._stream() == 103
