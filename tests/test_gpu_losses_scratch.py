"""The losses that have scratch memory do not depend on what it held, on any of their routes"""
import pytest
import torch

from loss_cases import DEV, TORCH

pytestmark = pytest.mark.gpu


def _same_with_any_scratch(op, call):
    want = [x.clone() for x in call()]
    gen = torch.Generator(device=DEV).manual_seed(0)
    for fill in (lambda w: w.fill_(255), lambda w: w.zero_(), lambda w: w.random_(0, 256, generator=gen)):
        assert op._scratch
        for w in op._scratch.values():
            fill(w)
        assert all(torch.equal(a, b) for a, b in zip(call(), want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(9, 301, 5), (9, 20001, 300), (600, 20001, 70), (33000, 40, 5), (7, 140001, 256)])
def test_distillation(rows, vocab, top, rest, dtype):
    from paper_2504_03662_amd.loss_ops import DeviceDistillation
    torch.manual_seed(rows)
    z = (2 * torch.randn(rows, vocab, device=DEV)).to(TORCH[dtype])
    at, tl = torch.randint(-1, vocab, (rows, top), device=DEV), torch.randn(rows, top, device=DEV)
    w = torch.rand(rows, device=DEV)
    w[::3] = 0.0
    at[1] = -1
    op = DeviceDistillation(vocab, dtype)
    _same_with_any_scratch(op, lambda: op.forward_backward(z, at, tl, torch.full_like(w, 9.0) if rest else None, w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(9, 301), (9, 20001), (1100, 301), (7, 140001)])
def test_preference(rows, vocab, dtype):
    from paper_2504_03662_amd.loss_ops import DevicePreferenceLoss
    torch.manual_seed(rows)
    z, ids = (2 * torch.randn(rows, vocab, device=DEV)).to(TORCH[dtype]), torch.randint(-1, vocab, (rows,), device=DEV)
    w = torch.rand(rows, device=DEV)
    w[::3] = 0.0
    starts = torch.tensor([1, 3, 3, 5, rows - 1], dtype=torch.int32, device=DEV)
    op = DevicePreferenceLoss(vocab, dtype)
    _same_with_any_scratch(op, lambda: op.forward_backward(z, ids, starts, None, w))
