"""Losses of logits where they take other launches than for a few rows: teachers that a launch of their own reads, pairs that are added up
in one, and entries that need more than 64 KB of LDS."""
import math

import pytest
import torch

import test_gpu_losses as few
from loss_cases import DEV, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["holes", "twice"])
@pytest.mark.parametrize("top,size", [(3, (300, 100, 5, 3)), (64, (257, 1001, 3, 1)), (65, (301, 1000, 0, 0)), (1024, (258, 2048, 0, 0)),
                                      (1024, (5, 2048, 0, 0)), (1000, (6, 1001, 1, 0)), (256, (259, 16400, 0, 0))], ids=str)
def test_distillation(top, size, kind, rest, dtype):
    few.test_distillation(top, size, kind, rest, dtype)


@pytest.mark.parametrize("dtype,rest,top,size", [("bf16", True, 64, (515, 16400, 0, 0)), ("f32", False, 65, (513, 8300, 4, 0)),
                                                 ("bf16", False, 256, (2049, 4800, 0, 0)), ("f32", True, 9, (2051, 2200, 0, 0)),
                                                 ("bf16", True, 66, (32769, 70, 0, 0)), ("f32", False, 5, (32771, 19, 2, 1))], ids=str)
def test_distillation_of_so_many_rows_that_a_launch_reads_the_teachers(dtype, rest, top, size):
    few.test_distillation(top, size, "twice", rest, dtype)


@pytest.mark.parametrize("name", ["distill", "rest"])
def test_captured_with_a_launch_for_the_teachers(name):
    rows, vocab = 600, 17000
    call = few._calls(vocab, "bf16", rows)[name]
    z = (2 * torch.randn(rows, vocab, device=DEV)).bfloat16()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    call(z)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = call(z)
    for _ in range(3):
        z.copy_((2 * torch.randn(rows, vocab, device=DEV)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        assert few._same(out, call(z))


@pytest.mark.parametrize("name", few.NAMES)
def test_captured_and_replayed(name):
    """Replays with other logits between eager calls of the same object, on the same stream"""
    rows, vocab = 1100, 301
    call = few._calls(vocab, "bf16", rows)[name]
    z = (2 * torch.randn(rows, vocab, device=DEV)).bfloat16()
    call(z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call(z)
    for _ in range(4):
        z.copy_((2 * torch.randn(rows, vocab, device=DEV)).bfloat16())
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            eager = call(z)
        torch.cuda.synchronize()
        assert few._same(out, eager)


def test_captured_with_much_lds():
    """The launch asks for more LDS than a kernel has unasked, the first time inside of a capture"""
    rows, vocab, top = 9, 2000, 1024
    op = few._ops().DeviceDistillation(vocab, "f32", scale=0.5)
    at = torch.stack([torch.randperm(vocab, device=DEV)[:top] for _ in range(rows)])
    tl, z = torch.randn(rows, top, device=DEV), torch.randn(rows, vocab, device=DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = op.forward_backward(z, at, tl)
    for _ in range(3):
        z.copy_(torch.randn(rows, vocab, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert few._same(out, op.forward_backward(z, at, tl))


@pytest.mark.parametrize("name", [n for n in few.NAMES if n != "preference"])
@pytest.mark.parametrize("vocab", [301, 3001])
def test_rows_do_not_depend_on_their_neighbours(name, vocab):
    """Rows that follow 1100 others have the same gradient as on their own, where the loss is a row's"""
    rows = 1100
    z = (2 * torch.randn(rows, vocab, device=DEV)).bfloat16()
    call = few._calls(vocab, "bf16", rows)[name]
    first = call(z)
    other = z.clone()
    other[:-3] = torch.randn(rows - 3, vocab, device=DEV).bfloat16()
    second = call(other)
    assert all(torch.equal(a[-3:], b[-3:]) for a, b in zip(first, second))


@pytest.mark.parametrize("dtype,vocab", [("bf16", 1001), ("f32", 1001), ("bf16", 20000), ("bf16", 140001)])
def test_masked_with_the_lowest_value(dtype, vocab):
    """Columns of the type's lowest number have no probability; a row of nothing else is uniform"""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = (2 * torch.randn(5, vocab, device=DEV)).to(t)
    low = torch.finfo(t).min
    z[:, vocab // 2:] = low
    z[4] = low
    ids = torch.tensor([0, 1, 2, 3, vocab - 1], device=DEV)
    op = few._ops().DeviceTokenLoss(vocab, dtype)
    loss, dz = op.forward_backward(z, ids)
    cut = op.__class__(vocab // 2, dtype).forward_backward(z[:, :vocab // 2].contiguous(), ids.clamp(max=vocab // 2 - 1))
    # the same numbers in another order: the log sum's bound twice, losses of about 10
    bound = 2 * (few.delta(vocab) + 20 * few.U)
    assert float((loss[:4] - cut[0][:4]).abs().max()) <= bound
    assert not dz[:4, vocab // 2:].any()
    step = 2 * few.HALF_STEP[dtype]
    assert float((dz[:4, :vocab // 2].float() - cut[1][:4].float()).abs().max()) <= step + 2 * bound
    assert abs(float(loss[4]) - math.log(vocab)) <= bound
    assert abs(float(dz[4, 0]) * vocab - 1.0) <= step + 2 * bound
    policy = few._ops().DevicePolicyLoss(vocab, dtype).forward_backward(z, ids, -loss, torch.ones(5, device=DEV))
    assert all(bool(torch.isfinite(x).all()) for x in policy)
    top = dev(torch.arange(8).repeat(5, 1), torch.int64)
    for lse in (None, torch.full((5,), 9.0, device=DEV)):
        got = few._ops().DeviceDistillation(vocab, dtype).forward_backward(z, top, torch.randn(5, 8, device=DEV), lse)
        assert all(bool(torch.isfinite(x).all()) for x in got)
