"""The operators around the block together, as a small decoder uses them: its gradient against differences of its loss, and the
task it is for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _model(**kw):
    from paper_2504_03662_amd.decoder_step import CopyingDecoder
    return CopyingDecoder(**kw)


def test_gradient_against_differences():
    """Along the gradient g of one group of weights the loss changes by 2 e |g|^2 between w + e g and w - e g; e makes that 0.04.
    The loss is about 20 and its fp32 arithmetic is off by 20 x 2^-24 x a few tens, 1e-4 of it by far at most: 2 % of the change.
    Terms of the third order in e are a change of 0.02 in a loss that varies on a scale of its own size: (0.02 / 20)^2.  Together
    3 %."""
    model = _model(vocab=19, batch=3, length=11, hidden=128, heads=4, key_heads=2, dtype="f32")
    data = model.batch_of(3)
    model.train_step(*data, lr=0.0)
    grads = {n: w.grad.clone() for n, w in model.weights.items()}
    for names in (["table"], ["wq", "wk"], ["gain_q", "gain_k"], ["wv", "wo"], ["w_qkv", "w_o", "w_fc1", "w_fc2", "b_fc2"]):
        square = sum(float((grads[n].double() ** 2).sum()) for n in names)
        e = 0.02 / square
        loss = []
        for sign in (1.0, -1.0):
            for n in names:
                w = model.weights[n]
                w.value.add_(grads[n].view_as(w.value), alpha=sign * e)
            loss.append(float(model.train_step(*data, lr=0.0)))      # the step writes the copies back from the masters
        assert abs(loss[0] - loss[1] - 0.04) <= 0.03 * 0.04, (names, loss, square)


def test_learns_to_copy_and_reads_one_token_at_a_time():
    from paper_2504_03662_amd.decoder_step import copied
    model = _model()
    losses = [float(model.train_step(*model.batch_of(i))) for i in range(120)]
    assert max(losses[-10:]) < 0.1 * losses[0], losses[::10]
    src, lens, inp = model.batch_of(10 ** 6)
    assert copied(src, lens, model.decode(src, lens)) >= 0.95
    # one token at a time and all at once read the same: o is rounded to 8 bits once in both
    source = model.read_source(src)
    f = model.forward(inp, source, lens)
    at = torch.full((model.batch, 1), 5, dtype=torch.int32, device=model.device)
    qn, _ = model.norm.forward(f["q"][:, 5:6], None, model.value("gain_q"), None, model.cos, model.sin, at)
    assert torch.equal(qn, f["qn"][:, 5:6])
    o, _ = model.cross.forward(qn, source[2], source[3], lens)
    scale = float(source[3].float().abs().max())
    assert float((o.float() - f["o"][:, 5:6].float()).abs().max()) <= 2 ** -7 * scale
