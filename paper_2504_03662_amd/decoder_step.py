"""A small decoder that reads an encoder's states, trained and then read from one token at a time: token embedding -> causal
block -> normed and rotated queries and keys -> cross attention -> the embedding table as output layer.

The task is to copy a ragged source that stands there in full, so the decoder can only know the next token by looking at the right
position of the source.  Every operator is the library's (`DeviceEmbedding`, `DeviceLayer`, `DeviceHeadNorm`,
`DeviceCrossAttention`, `adamw_step`); the projections and the loss are a few lines of torch.  The losses of `loss_ops` take that
loss's place with --learn: `tokens` from the start, the others for a second half of the steps, after a first half of `train_step`s.
`distill` trains another decoder from the first one's top logits, `policy` rewards drawn tokens that are the source's, `prefer`
prefers the source to the same with a few wrong tokens.

    python -m paper_2504_03662_amd.decoder_step [--steps 200] [--learn tokens|distill|policy|prefer]
"""
from __future__ import annotations

import argparse

import torch

from . import binding as gx, inputs as I
from .decoder_ops import DeviceCrossAttention, DeviceEmbedding, DeviceHeadNorm
from .loss_ops import DeviceDistillation, DevicePolicyLoss, DevicePreferenceLoss, DeviceTokenLoss
from .runtime import DeviceLayer

START = 1                                           # first decoder token; 0 pads
THETA = 10000.0


class Weight:
    """fp32 master, AdamW moments and gradient of a parameter, and the copy that the kernels read."""

    def __init__(self, value, dtype):
        self.master = value.to(torch.float32, copy=True)
        self.m, self.v, self.grad = (torch.zeros_like(self.master) for _ in range(3))
        self.value = self.master.to(dtype, copy=True)

    def step(self, t, lr, stream):
        gx.adamw_step(self.master.numel(), self.master, self.m, self.v, self.grad, self.value,
                      gx.GX_BF16 if self.value.dtype == torch.bfloat16 else gx.GX_F32, step=t, lr=lr, stream=stream)


class CopyingDecoder:
    def __init__(self, vocab=64, batch=8, length=32, hidden=512, heads=4, key_heads=2, dtype="bf16", device="cuda:0", seed=0):
        self.vocab, self.batch, self.length, self.hidden, self.heads, self.key_heads = vocab, batch, length, hidden, heads, key_heads
        self.device, self.head_dim = device, hidden // heads
        shape = I.LayerShape(hidden, heads, 2 * hidden, seq=length, micro_batch=batch, dtype=dtype)
        self.layer = DeviceLayer(shape, I.full_params(shape, case=seed), device)
        self.embed = DeviceEmbedding(vocab, hidden, dtype, scale=hidden ** 0.5, pad_id=0, device=device)
        self.norm = DeviceHeadNorm(self.head_dim, self.head_dim, dtype, device=device)
        self.cross = DeviceCrossAttention(self.head_dim, dtype, device=device)
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape):
            return (torch.randn(shape, generator=gen) * hidden ** -0.5).to(device)

        kv = key_heads * self.head_dim
        self.weights = {"table": normal(vocab, hidden), "wq": normal(hidden, hidden), "wk": normal(hidden, kv),
                        "wv": normal(hidden, kv), "wo": normal(hidden, hidden),
                        "gain_q": torch.ones(self.head_dim, device=device), "gain_k": torch.ones(self.head_dim, device=device)}
        self.weights = {n: Weight(w, self.layer.tdtype) for n, w in self.weights.items()}
        for n, p in self.layer.params.items():                    # the block's: its gradients are the layer's own
            w = self.weights[n] = Weight(p, p.dtype)
            w.value, w.grad = p, self.layer.grads[n]
        angle = torch.arange(length).double()[:, None] * THETA ** (-torch.arange(self.head_dim // 2).double() * 2 / self.head_dim)
        self.cos, self.sin = angle.cos().float().to(device), angle.sin().float().to(device)
        self.t = 0
        logits = dict(dtype="f32", device=device)
        self.token_loss = DeviceTokenLoss(vocab, ignore_id=0, **logits)
        self.policy_loss = DevicePolicyLoss(vocab, kl=0.05, ignore_id=0, **logits)
        self.preference_loss = DevicePreferenceLoss(vocab, ignore_id=0, **logits)
        self.distillation = DeviceDistillation(vocab, **logits)

    def batch_of(self, seed):
        """(source ids, source lengths, decoder inputs): sources of different lengths, the rest of a row is padding"""
        gen = torch.Generator().manual_seed(seed)
        lens = torch.randint(self.length // 2, self.length + 1, (self.batch,), generator=gen, dtype=torch.int32)
        src = torch.randint(2, self.vocab, (self.batch, self.length), generator=gen)
        src[torch.arange(self.length)[None, :] >= lens[:, None]] = 0
        inp = torch.cat([torch.full((self.batch, 1), START), src[:, :-1]], dim=1)
        return src.to(self.device), lens.to(self.device), inp.to(self.device)

    def value(self, name):
        return self.weights[name].value

    def _heads(self, x, n):
        return x.view(self.batch, -1, n, self.head_dim)

    def read_source(self, src):
        """What a decoder keeps of a source: its states, and its keys, as projected and as normed and rotated, and values"""
        states = self.embed.forward(self.value("table"), src)
        k, v = (self._heads(states @ self.value(n), self.key_heads) for n in ("wk", "wv"))
        _, kn = self.norm.forward(None, k, None, self.value("gain_k"), self.cos, self.sin)
        return states, k, kn, v

    def forward(self, inp, source, lens, want_lse=True):
        """All of the decoder's positions at once -> what the backward pass needs and the logits"""
        x = self.embed.forward(self.value("table"), inp).view(-1, self.hidden)
        h = self.layer.forward(x)["y"]
        q = self._heads(h @ self.value("wq"), self.heads)
        qn, _ = self.norm.forward(q, None, self.value("gain_q"), None, self.cos, self.sin)
        o, lse = self.cross.forward(qn, source[2], source[3], lens, want_lse=want_lse)
        y = h + o.view(-1, self.hidden) @ self.value("wo")
        return dict(x=x, h=h, q=q, qn=qn, o=o, lse=lse, y=y, logits=y.float() @ self.value("table").float().t())

    def train_step(self, src, lens, inp, lr=2e-3):
        source = states, k, kn, v = self.read_source(src)
        f = self.forward(inp, source, lens)
        target = src.view(-1)
        logp = torch.log_softmax(f["logits"], dim=1)
        counts = target != 0
        loss = -(logp.gather(1, target[:, None])[:, 0] * counts).sum() / counts.sum()
        dlogits = logp.exp()
        dlogits.scatter_add_(1, target[:, None], torch.full_like(dlogits[:, :1], -1.0))
        dlogits *= (counts / counts.sum())[:, None]
        self._update(source, src, lens, inp, f, dlogits, lr)
        return loss

    def _update(self, source, src, lens, inp, f, dlogits, lr):
        """From the gradient of the logits to the weights"""
        states, k, kn, v = source
        w, flat = self.weights, (lambda x: x.reshape(x.shape[0] * x.shape[1], -1))
        table = w["table"].value.float()
        w["table"].grad.copy_(dlogits.t() @ f["y"].float())
        dy = (dlogits @ table).to(f["y"].dtype)
        o = f["o"].view(-1, self.hidden)
        w["wo"].grad.copy_(o.float().t() @ dy.float())
        do = (dy @ w["wo"].value.t()).view_as(f["o"])
        dqn, dkn, dv = self.cross.backward(f["qn"], kn, v, f["o"], f["lse"], do, lens)
        gains, angles = (w["gain_q"].value, w["gain_k"].value), (self.cos, self.sin)
        dq, dk, _, _ = self.norm.backward(f["q"], k, dqn, dkn, *gains, *angles, dgain_q=w["gain_q"].grad, dgain_k=w["gain_k"].grad)
        dq, dk, dv, s = flat(dq), flat(dk), flat(dv), flat(states)
        w["wq"].grad.copy_(f["h"].float().t() @ dq.float())
        w["wk"].grad.copy_(s.float().t() @ dk.float())
        w["wv"].grad.copy_(s.float().t() @ dv.float())
        dstates = dk @ w["wk"].value.t() + dv @ w["wv"].value.t()
        dh = dy + dq @ w["wq"].value.t()
        dx = self.layer.backward(f["x"], dh)
        # one table for the output layer, the decoder's inputs and the source
        self.embed.backward(inp, dx.view(*inp.shape, -1), out=w["table"].grad, accumulate=True)
        self.embed.backward(src, dstates.view(*src.shape, -1), out=w["table"].grad, accumulate=True)
        self.t += 1
        for x in w.values():
            x.step(self.t, lr, torch.cuda.current_stream().cuda_stream)

    def learn(self, objective, src, lens, inp, lr=2e-3):
        """A step with an objective: logits [batch, length, vocab] -> (losses, their sum's gradient by the logits) -> the losses' sum"""
        source = self.read_source(src)
        f = self.forward(inp, source, lens)
        losses, dlogits = objective(f["logits"].view(*inp.shape, -1))
        self._update(source, src, lens, inp, f, dlogits.view(-1, self.vocab), lr)
        return losses.sum()

    def take_weights(self, other):
        for n, w in self.weights.items():
            w.master.copy_(other.weights[n].master)
            w.value.copy_(other.weights[n].value)

    def logits(self, src, lens, inp):
        return self.forward(inp, self.read_source(src), lens, want_lse=False)["logits"].view(*inp.shape, -1)

    # Objectives.  Gradients are written over the logits.
    def _mean(self, ids):
        counts = (ids != 0).float()
        return counts / counts.sum()

    def tokens(self, src):
        """Cross entropy"""
        return lambda z: self.token_loss.forward_backward(z, src, self._mean(src), out=z)

    def distill(self, src, teacher_logits, top=8):
        """What another decoder has told of itself: its top logits, and their distance from its log sum"""
        best, ids = teacher_logits.topk(top, dim=2)
        _, lse = self.token_loss.logp(teacher_logits, src)
        return lambda z: self.distillation.forward_backward(z, ids, best, lse, self._mean(src), out=z)

    def policy(self, src, drawn, old_logp, ref_logp):
        """Tokens that an older policy has drawn, and its log probabilities: those that are the source's are to come more often"""
        right = (drawn == src).float()
        advantages = right - (right * self._mean(src)).sum()

        def objective(z):
            losses, _, dlogits = self.policy_loss.forward_backward(z, drawn, old_logp, advantages, ref_logp, self._mean(src), out=z)
            return losses, dlogits
        return objective

    def prefer(self, ids, ref_logp):
        """Samples 2 i and 2 i + 1 are chosen and rejected answers to one source"""
        starts = torch.arange(self.batch + 1, dtype=torch.int32, device=self.device) * self.length
        each = torch.full((self.batch // 2,), 2.0 / self.batch, device=self.device)

        def objective(z):
            losses, _, dlogits = self.preference_loss.forward_backward(z, ids, starts, ref_logp, None, each, out=z)
            return losses, dlogits
        return objective

    def drawn_from(self, src, lens, inp, seed):
        """A token of every position, drawn after the source's tokens before it -> (tokens, their log probabilities)"""
        z = self.logits(src, lens, inp)
        gen = torch.Generator().manual_seed(seed)
        p = torch.softmax(z, dim=2).cpu().view(-1, self.vocab)
        drawn = torch.multinomial(p, 1, generator=gen).view(src.shape).to(self.device)
        drawn = torch.where(src == 0, 0, drawn)
        return drawn, self.token_loss.logp(z, drawn)[0]

    def pairs_of(self, seed):
        """(sources, lengths, decoder inputs, answers): every source twice, answered by itself and by a copy with wrong tokens"""
        src, lens, _ = self.batch_of(seed)
        src, lens = src[:self.batch // 2].repeat_interleave(2, dim=0), lens[:self.batch // 2].repeat_interleave(2)
        gen = torch.Generator().manual_seed(seed + 1)
        wrong = torch.rand(src.shape, generator=gen) < 0.2
        wrong[0::2] = False
        other = torch.randint(2, self.vocab, src.shape, generator=gen)
        ids = torch.where(wrong.to(self.device) & (src != 0), other.to(self.device), src)
        inp = torch.cat([torch.full_like(ids[:, :1], START), ids[:, :-1]], dim=1)
        return src, lens, inp, ids

    def decode(self, src, lens):
        """Greedy: the source's keys and values stay as they are, and each step's queries are one token of every sample"""
        source = self.read_source(src)
        inp = torch.zeros_like(src)
        inp[:, 0] = START
        out = torch.zeros_like(src)
        for i in range(self.length):
            x = self.embed.forward(self.value("table"), inp).view(-1, self.hidden)
            h = self.layer.forward(x)["y"].view(self.batch, self.length, -1)[:, i]
            q = self._heads(h @ self.value("wq"), self.heads)
            at = torch.full((self.batch, 1), i, dtype=torch.int32, device=self.device)
            qn, _ = self.norm.forward(q, None, self.value("gain_q"), None, self.cos, self.sin, at)
            o, _ = self.cross.forward(qn, source[2], source[3], lens, want_lse=False)
            y = h + o.view(self.batch, -1) @ self.value("wo")
            out[:, i] = (y.float() @ self.value("table").float().t()).argmax(dim=1)
            if i + 1 < self.length:
                inp[:, i + 1] = out[:, i]
        return out


def copied(src, lens, out):
    """Share of the source's tokens that came out"""
    counts = torch.arange(src.shape[1], device=src.device)[None, :] < lens[:, None]
    return float(((src == out) & counts).sum() / counts.sum())


def taught(model, first, how, seed, lr):
    """A step of an objective of `loss_ops` on a batch; `first` is the teacher, or what the decoder is held near"""
    if how == "prefer":
        src, lens, inp, ids = model.pairs_of(seed)
        objective = model.prefer(ids, first.token_loss.logp(first.logits(src, lens, inp), ids)[0])
        return model.learn(objective, src, lens, inp, lr)
    data = src, _, _ = model.batch_of(seed)
    if how == "tokens":
        objective = model.tokens(src)
    elif how == "distill":
        objective = model.distill(src, first.logits(*data))
    else:
        drawn, old_logp = model.drawn_from(*data, seed)
        objective = model.policy(src, drawn, old_logp, first.token_loss.logp(first.logits(*data), drawn)[0])
    return model.learn(objective, *data, lr)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--learn", choices=("tokens", "distill", "policy", "prefer"))
    a = ap.parse_args()
    model = first = CopyingDecoder()
    half = 0 if a.learn == "tokens" else a.steps // 2
    for i in range(a.steps):
        if a.learn and i == half > 0:
            model = CopyingDecoder(seed=1)
            if a.learn != "distill":
                model.take_weights(first)
        if a.learn and i >= half:
            loss = taught(model, first, a.learn, i, 2e-4 if a.learn in ("policy", "prefer") else 2e-3)
        else:
            loss = model.train_step(*model.batch_of(i))
        if i % 20 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss):.4f}", flush=True)
    src, lens, _ = model.batch_of(10 ** 6)
    print(f"read back one token at a time: {100 * copied(src, lens, model.decode(src, lens)):.1f} % of an unseen batch")


if __name__ == "__main__":
    main()
