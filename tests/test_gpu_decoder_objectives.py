"""The losses of logits where a small decoder learns from them: the gradient of every weight against differences of the loss, the
gradient of cross entropy against the decoder's own, and steps of each."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
OBJECTIVES = ("tokens", "distill", "policy", "prefer")


def _model(**kw):
    from paper_2504_03662_amd.decoder_step import CopyingDecoder
    return CopyingDecoder(**{**dict(vocab=19, batch=4, length=11, hidden=128, heads=4, key_heads=2, dtype="f32"), **kw})


def _objective(model, first, how):
    """(the objective, its batch), with what others say held fixed.  Two decoders that have learnt nothing say much the same (their loss is
    0.02) and are sure of it (what they draw has next to no gradient): the teacher is a table of random logits, and the drawn tokens
    are any."""
    if how == "prefer":
        src, lens, inp, ids = model.pairs_of(3)
        return model.prefer(ids, first.token_loss.logp(first.logits(src, lens, inp), ids)[0]), (src, lens, inp)
    data = src, _, _ = model.batch_of(3)
    if how == "tokens":
        return model.tokens(src), data
    if how == "distill":
        gen = torch.Generator().manual_seed(7)
        return model.distill(src, (8.0 * torch.randn(*src.shape, model.vocab, generator=gen)).to(model.device)), data
    gen = torch.Generator().manual_seed(5)
    drawn = torch.where(src == 0, 0, torch.randint(2, model.vocab, src.shape, generator=gen).to(model.device))
    drawn[:, ::3] = src[:, ::3]                                      # some of them right
    old_logp, _ = model.token_loss.logp(model.logits(*data), drawn)
    return model.policy(src, drawn, old_logp, first.token_loss.logp(first.logits(*data), drawn)[0]), data


@pytest.mark.parametrize("how", OBJECTIVES)
def test_gradient_against_differences(how):
    """Along the gradient g of one group of weights the loss changes by 2 e |g|^2 between w + e g and w - e g; e makes that 2^-9 of
    the loss's own scale S: 20 for cross entropy and distillation (a decoder that has learnt nothing is off by logits of about
    20), 1 for the policy's and the preference's, whose derivative by a log probability is at most a token's weight.  A logit
    is off by 20 x 2^-24 x a few tens, 3e-5: of the change 3e-5 / 2^-9, 1.5 %, if every token were off to the same side.  Terms of the third
    order in e: (2^-10)^2 on a scale of S.  Together 3 %.  The clip is far away: its own gradient is tested with the operator."""
    model, first = _model(), _model(seed=1)
    model.policy_loss.clip_low, model.policy_loss.clip_high = 0.99, 1e3
    objective, data = _objective(model, first, how)
    model.learn(objective, *data, lr=0.0)
    grads = {n: w.grad.clone() for n, w in model.weights.items()}
    change = (20.0 if how in ("tokens", "distill") else 1.0) * 2.0 ** -9
    for names in (["table"], ["wq", "wk"], ["gain_q", "gain_k"], ["wv", "wo"], ["w_qkv", "w_o", "w_fc1", "w_fc2", "b_fc2"]):
        square = sum(float((grads[n].double() ** 2).sum()) for n in names)
        e = change / 2 / square
        loss = []
        for sign in (1.0, -1.0):
            for n in names:
                w = model.weights[n]
                w.value.add_(grads[n].view_as(w.value), alpha=sign * e)
            loss.append(float(model.learn(objective, *data, lr=0.0)))     # the step writes the copies back from the masters
        assert abs(loss[0] - loss[1] - change) <= 0.03 * change, (names, loss, square)


def _plain(model, how, z, objective):
    """The objective's loss in 64 bits, from what it holds"""
    held = dict(zip(objective.__code__.co_freevars, (c.cell_contents for c in objective.__closure__)))
    logp = torch.log_softmax(z, dim=2)
    at = lambda ids: logp.gather(2, ids[..., None])[..., 0]
    if how == "tokens":
        return -(at(held["src"]) * model._mean(held["src"]).double()).sum()
    if how == "distill":
        q = (held["best"].double() - held["lse"].double()[..., None]).exp()
        here = logp.gather(2, held["ids"])
        rest = (1.0 - q.sum(2)).clamp(min=0.0)
        others = logp.scatter(2, held["ids"], -math.inf).logsumexp(2)           # 1 - sum of p, without the difference
        loss = (q * (q.log() - here)).sum(2) + torch.where(rest > 0, rest * (rest.clamp(min=1e-300).log() - others), 0.0)
        return (loss * model._mean(held["src"]).double()).sum()
    if how == "policy":
        drawn, loss = held["drawn"], model.policy_loss
        own, adv = at(drawn), held["advantages"].double()
        r, d = (own - held["old_logp"].double()).exp(), held["ref_logp"].double() - own
        gain = torch.minimum(r * adv, r.clamp(1 - loss.clip_low, 1 + loss.clip_high) * adv)
        return ((-gain + loss.kl * (d.exp() - d - 1)) * model._mean(held["src"]).double() * (drawn != 0)).sum()
    ids, loss = held["ids"], model.preference_loss
    reward = loss.beta * ((at(ids) - held["ref_logp"].double()) * (ids != 0)).sum(1)
    return (-torch.nn.functional.logsigmoid(reward[0::2] - reward[1::2]) * held["each"].double()).sum()


@pytest.mark.parametrize("how", OBJECTIVES)
def test_gradient_is_the_formulas(how):
    """The weights' gradients are linear in the logits', whose entries are off by a few fp32 roundings of exponentials of numbers up to
    40, 40 x 2^-24 x 4 = 2^-17: 2^-16 of the gradient's norm leaves a factor of 2, and the loss's own 2^-16 too.  A policy whose
    old_logp is its own has ratios of 1, and half of its tokens' gains cancel: its norm is not small, its loss is, so that the
    loss is measured against the sizes of its terms, at most 1."""
    model, first = _model(), _model(seed=1)
    objective, data = _objective(model, first, how)
    z = model.logits(*data).double().requires_grad_()
    plain = _plain(model, how, z, objective)
    plain.backward()
    plain = plain.detach()
    model.learn(lambda _: (plain, z.grad.float()), *data, lr=0.0)
    grads = {n: w.grad.clone() for n, w in model.weights.items()}
    loss = float(model.learn(objective, *data, lr=0.0))
    assert abs(loss - float(plain)) <= 2.0 ** -16 * max(1.0, abs(float(plain)))
    for n, w in model.weights.items():
        assert float((w.grad - grads[n]).norm()) <= 2.0 ** -16 * float(grads[n].norm()), n


def test_tokens_are_the_decoders_own_loss():
    """Cross entropy of the operator and of the decoder's own lines: logits alike bit by bit, both gradients dlogits within a few
    fp32 roundings of p - 1 at the token (exp and log of numbers up to 40: 40 x 2^-24 x 4), and the weights' gradients linear in dlogits:
    2^-16 of their norm leaves a factor of 1.6."""
    model = _model()
    data = model.batch_of(3)
    own = float(model.train_step(*data, lr=0.0))
    grads = {n: w.grad.clone() for n, w in model.weights.items()}
    loss = float(model.learn(model.tokens(data[0]), *data, lr=0.0))
    assert abs(loss - own) <= 2.0 ** -16 * abs(own)
    for n, w in model.weights.items():
        assert float((w.grad - grads[n]).norm()) <= 2.0 ** -16 * float(grads[n].norm()), n


@pytest.mark.parametrize("how", OBJECTIVES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps(how, dtype):
    """Steps run one after another, change every weight, and leave all of them finite"""
    from paper_2504_03662_amd.decoder_step import taught
    model, first = (_model(dtype=dtype, vocab=64, batch=8, length=32, hidden=512, seed=i) for i in range(2))
    if how != "distill":
        model.take_weights(first)
    before = {n: w.master.clone() for n, w in model.weights.items()}
    for seed in range(3):
        assert math.isfinite(float(taught(model, first, how, seed, 1e-3)))
    for n, w in model.weights.items():
        assert torch.isfinite(w.master).all(), n
        if n != "b_qkv":                                            # of whom the keys' third has no gradient
            assert not torch.equal(w.master, before[n]), n
