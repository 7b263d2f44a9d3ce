"""What a decoder learns from, on torch tensors: log probabilities of tokens and cross entropy, the clipped policy loss, the preference
loss of pairs of sequences and distillation from a teacher's top logits, each with the gradient of the logits.  Plumbing like
`decoder_ops`, and of the same manner: calls work on the current stream and return without waiting, shapes and types are checked
here, outputs are new tensors unless `out` is given.

Logits are [..., vocab] with one distance between rows: contiguous, or a view of the first columns of a padded matrix.  Everything
that belongs to a row (ids, weights, log probabilities) has the logits' shape without the last one.  Gradients may be written over
the logits (`out=logits`).  Losses come by row or pair, already multiplied by the weights: their sum is the batch's loss, and with
weights of mask / mask.sum() its mean."""
from __future__ import annotations

import torch

from . import binding as gx
from .decoder_ops import _need, _Operator


_ID_BYTES = {torch.int32: 4, torch.int64: 8}


class _LogitsOperator(_Operator):
    """Sizes and checks of an operator on logits"""

    def __init__(self, vocab, dtype, scale, ignore_id, first_id, whole_vocab, device):
        super().__init__(dtype, device)
        self.vocab, self.scale, self.ignore_id, self.first_id, self.whole_vocab = vocab, scale, ignore_id, first_id, whole_vocab

    def _rows(self, name, t, shape=None):
        """The distance between the rows of a tensor of logits"""
        if t.is_contiguous() and t.dtype is self.tdtype and t.get_device() == self.index and t.dim() > 1 and t.shape[-1] == self.vocab and (
                shape is None or t.shape == shape):
            return self.vocab
        if shape is None:
            shape = t.shape
            _need(len(shape) > 1 and shape[-1] == self.vocab, f"{name}: not [..., {self.vocab}]")
        self._check(name, t, shape, self.tdtype, False)
        st = t.stride()
        _need(st[-1] == 1 or self.vocab == 1, f"{name}: columns are not contiguous")
        # dimensions of one row have no distance that counts
        dims = [(n, d) for n, d in zip(shape[:-1], st[:-1]) if n != 1]
        _need(all(a == n * b for (_, a), (n, b) in zip(dims, dims[1:])), f"{name}: no one distance between rows")
        stride = dims[-1][1] if dims else self.vocab
        _need(stride >= self.vocab, f"{name}: rows overlap")
        return stride

    def _gradient(self, logits, stride, out):
        """(where the gradient goes, the distance of its rows): `out`, or a new tensor whose rows lie as the logits' do"""
        if out is not None:
            return out, self._rows("out", out, logits.shape)
        begin = logits.data_ptr() % 16
        if stride == self.vocab and begin == 0:
            return torch.empty_like(logits, memory_format=torch.contiguous_format), stride
        per = 8 if self.tdtype == torch.bfloat16 else 4             # elements of 16 bytes
        begin //= 16 // per
        stride = self.vocab + (stride - self.vocab) % per
        flat = torch.empty(logits.numel() // self.vocab * stride + begin, dtype=self.tdtype, device=self.device)
        strides, step = [1], stride
        for n in reversed(logits.shape[:-1]):
            strides.append(step)
            step *= n
        return flat.as_strided(logits.shape, strides[::-1], begin), stride

    def _by_row(self, name, t, shape):
        if t is not None:
            self._check(name, t, shape, torch.float32)

    def _ids(self, ids, shape):
        id_bytes = _ID_BYTES.get(ids.dtype)
        if id_bytes is None:
            raise ValueError(f"ids: {ids.dtype}, not int32 or int64")
        self._check("ids", ids, shape, ids.dtype)
        return id_bytes

    def _cfg(self, rows, id_bytes, stride, grad_stride):
        return gx.LogitsCfg(rows, self.vocab, self.gtype, id_bytes, 0, self.scale, stride, grad_stride, self.first_id, self.whole_vocab,
                            self.ignore_id)


class DeviceTokenLoss(_LogitsOperator):
    """Log probabilities of tokens under softmax(scale * logits), and cross entropy.  Rows whose id is `ignore_id` do not count.  A rank
    that holds columns [first_id, first_id + vocab) of whole_vocab has `logp` and `logp_backward`."""

    def __init__(self, vocab, dtype="bf16", scale=1.0, ignore_id=-1, first_id=0, whole_vocab=None, device="cuda:0"):
        super().__init__(vocab, dtype, scale, ignore_id, first_id, first_id + vocab if whole_vocab is None else whole_vocab, device)

    def logp(self, logits, ids):
        """logits [..., vocab], ids [...] -> (logp, lse), fp32.  Over a shard lse is the shard's, and logp -lse where the token is another
        shard's: of the whole vocabulary lse = logsumexp of all lse, logp = sum of all (logp + lse) - lse.  A shard that has nothing but -inf in a
        row has lse = -inf and logp without it, which goes into the sum alone: logp + lse.masked_fill(lse == -inf, 0)."""
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        cfg = self._cfg(ids.numel(), self._ids(ids, shape), stride, stride)
        logp = self._new(shape, torch.float32)
        lse = torch.empty_like(logp)
        gx.logp_fwd(cfg, logits, ids, logp, lse, self._stream())
        return logp, lse

    def logp_backward(self, logits, ids, lse, dlogp, out=None):
        """lse of the whole vocabulary and the gradient of logp -> the gradient of the logits"""
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        id_bytes = self._ids(ids, shape)
        self._check("lse", lse, shape, torch.float32)
        self._check("dlogp", dlogp, shape, torch.float32)
        out, grad_stride = self._gradient(logits, stride, out)
        gx.logp_bwd(self._cfg(ids.numel(), id_bytes, stride, grad_stride), logits, ids, lse, dlogp, out, self._stream())
        return out

    def _run(self, logits, ids, weights, gradient, out):
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        id_bytes = self._ids(ids, shape)
        self._by_row("weights", weights, shape)
        out, grad_stride = self._gradient(logits, stride, out) if gradient else (None, stride)
        loss = self._new(shape, torch.float32) if weights is None else torch.empty_like(weights)
        gx.token_loss(self._cfg(ids.numel(), id_bytes, stride, grad_stride), logits, ids, weights, loss, None, out, self._stream())
        return loss, out

    def forward(self, logits, ids, weights=None):
        """weights fp32 [...] -> the rows' losses, -weight * logp"""
        return self._run(logits, ids, weights, False, None)[0]

    def forward_backward(self, logits, ids, weights=None, out=None):
        """-> (losses, the gradient of their sum by the logits), in one pass"""
        return self._run(logits, ids, weights, True, out)


class DevicePolicyLoss(_LogitsOperator):
    """The clipped policy loss of tokens that an older policy has drawn, with a KL term that holds the policy near a reference:
    weight * (-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl (exp(d) - d - 1)), r = exp(logp - old_logp), d = ref_logp - logp."""

    def __init__(self, vocab, dtype="bf16", clip_low=0.2, clip_high=0.2, kl=0.0, scale=1.0, ignore_id=-1, device="cuda:0"):
        super().__init__(vocab, dtype, scale, ignore_id, 0, vocab, device)
        self.clip_low, self.clip_high, self.kl = clip_low, clip_high, kl

    def _run(self, logits, ids, old_logp, advantages, ref_logp, weights, gradient, out):
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        id_bytes = self._ids(ids, shape)
        self._check("old_logp", old_logp, shape, torch.float32)
        self._check("advantages", advantages, shape, torch.float32)
        _need(ref_logp is not None or self.kl == 0, "kl: against which ref_logp?")
        self._by_row("ref_logp", ref_logp, shape)
        self._by_row("weights", weights, shape)
        out, grad_stride = self._gradient(logits, stride, out) if gradient else (None, stride)
        loss, logp = torch.empty_like(old_logp), torch.empty_like(old_logp)
        gx.policy_loss(self._cfg(ids.numel(), id_bytes, stride, grad_stride), gx.PolicyCfg(self.clip_low, self.clip_high, self.kl, 0),
                       gx.policy_in(old_logp, advantages, ref_logp, weights), logits, ids, loss, logp, out, self._stream())
        return loss, logp, out

    def forward(self, logits, ids, old_logp, advantages, ref_logp=None, weights=None):
        """fp32 [...] each, like ids -> (losses, logp)"""
        return self._run(logits, ids, old_logp, advantages, ref_logp, weights, False, None)[:2]

    def forward_backward(self, logits, ids, old_logp, advantages, ref_logp=None, weights=None, out=None):
        """-> (losses, logp, the gradient of the losses' sum by the logits), in one pass"""
        return self._run(logits, ids, old_logp, advantages, ref_logp, weights, True, out)


class DevicePreferenceLoss(_LogitsOperator):
    """The preference loss of pairs of sequences.  With x = beta (sum of weight * (logp - ref_logp) over the chosen sequence's rows - the
    same over the rejected one's) - margin it is -(1 - smoothing) log sigmoid(x) - smoothing log sigmoid(-x).  The rows of all
    sequences follow one another, chosen and rejected by turns: sequence j is rows starts[j] .. starts[j + 1] - 1."""

    def __init__(self, vocab, dtype="bf16", beta=0.1, margin=0.0, smoothing=0.0, scale=1.0, ignore_id=-1, device="cuda:0"):
        super().__init__(vocab, dtype, scale, ignore_id, 0, vocab, device)
        self.beta, self.margin, self.smoothing = beta, margin, smoothing

    def _pairs(self, rows, shape, starts, ref_logp, weights, pair_weights):
        _need(starts.dim() == 1 and starts.shape[0] % 2 == 1, "starts: not [2 * pairs + 1]")
        self._check("starts", starts, starts.shape, torch.int32)
        pairs = starts.shape[0] // 2
        self._by_row("ref_logp", ref_logp, shape)
        self._by_row("weights", weights, shape)
        self._by_row("pair_weights", pair_weights, (pairs,))
        return (pairs, gx.PairsCfg(pairs, rows, self.beta, self.margin, self.smoothing, 0),
                gx.pairs_in(starts, ref_logp, weights, pair_weights))

    def pairs(self, logp, starts, ref_logp=None, weights=None, pair_weights=None):
        """From log probabilities, fp32 of any shape -> (losses [pairs], rewards [2 * pairs], the gradient of the losses' sum by logp).  For
        logits in shards, between `DeviceTokenLoss.logp` and `logp_backward`."""
        self._check("logp", logp, logp.shape, torch.float32)
        n, cfg, inputs = self._pairs(logp.numel(), logp.shape, starts, ref_logp, weights, pair_weights)
        loss, rewards = self._new((n,), torch.float32), self._new((2 * n,), torch.float32)
        dlogp = self._new(logp.shape, torch.float32)
        gx.pairs_loss(cfg, inputs, logp, loss, rewards, dlogp, self._stream())
        return loss, rewards, dlogp

    def _run(self, logits, ids, starts, ref_logp, weights, pair_weights, gradient, out):
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        id_bytes = self._ids(ids, shape)
        n, pairs, inputs = self._pairs(ids.numel(), shape, starts, ref_logp, weights, pair_weights)
        out, grad_stride = self._gradient(logits, stride, out) if gradient else (None, stride)
        loss, rewards = self._new((n,), torch.float32), self._new((2 * n,), torch.float32)
        cfg, stream = self._cfg(ids.numel(), id_bytes, stride, grad_stride), self._stream()
        gx.preference_loss(cfg, pairs, inputs, logits, ids, loss, rewards, out,
                           self._workspace(gx.preference_workspace_bytes(cfg), stream), stream)
        return loss, rewards, out

    def forward(self, logits, ids, starts, ref_logp=None, weights=None, pair_weights=None):
        """starts int32 [2 * pairs + 1], ref_logp and weights fp32 like ids, pair_weights fp32 [pairs] -> (losses [pairs],
        rewards [2 * pairs])"""
        return self._run(logits, ids, starts, ref_logp, weights, pair_weights, False, None)[:2]

    def forward_backward(self, logits, ids, starts, ref_logp=None, weights=None, pair_weights=None, out=None):
        """-> (losses, rewards, the gradient of the losses' sum by the logits)"""
        return self._run(logits, ids, starts, ref_logp, weights, pair_weights, True, out)


class DeviceDistillation(_LogitsOperator):
    """KL divergence of softmax(scale * logits) from a teacher of whom each row has its top logits: q the softmax of scale * top_logits,
    or, with the teacher's own log sums, exp(scale * top_logits - top_lse), the other columns together being one more outcome."""

    def __init__(self, vocab, dtype="bf16", scale=1.0, device="cuda:0"):
        super().__init__(vocab, dtype, scale, -1, 0, vocab, device)

    def _run(self, logits, top_ids, top_logits, top_lse, weights, gradient, out):
        stride, shape = self._rows("logits", logits), logits.shape[:-1]
        _need(top_ids.shape[:-1] == shape and top_ids.dim() == logits.dim(), "top_ids: one dimension more than a row")
        id_bytes = self._ids(top_ids, top_ids.shape)
        _need(top_logits.dtype in (torch.float32, torch.bfloat16), f"top_logits: {top_logits.dtype}, not float32 or bfloat16")
        self._check("top_logits", top_logits, top_ids.shape, top_logits.dtype)
        self._by_row("top_lse", top_lse, shape)
        self._by_row("weights", weights, shape)
        out, grad_stride = self._gradient(logits, stride, out) if gradient else (None, stride)
        loss = self._new(shape, torch.float32) if weights is None else torch.empty_like(weights)
        distill = gx.DistillCfg(top_ids.shape[-1], gx.GX_BF16 if top_logits.dtype == torch.bfloat16 else gx.GX_F32, 0)
        cfg, stream = self._cfg(loss.numel(), id_bytes, stride, grad_stride), self._stream()
        gx.distill_loss(cfg, distill, gx.distill_in(top_ids, top_logits, top_lse, weights), logits, loss, out,
                        self._workspace(gx.distill_workspace_bytes(cfg, distill), stream), stream)
        return loss, out

    def forward(self, logits, top_ids, top_logits, top_lse=None, weights=None):
        """top_ids int32 or int64 [..., top] (-1: no entry), top_logits fp32 or bf16 [..., top], top_lse and weights fp32 [...] -> the
        rows' losses"""
        return self._run(logits, top_ids, top_logits, top_lse, weights, False, None)[0]

    def forward_backward(self, logits, top_ids, top_logits, top_lse=None, weights=None, out=None):
        """-> (losses, the gradient of their sum by the logits), in one pass"""
        return self._run(logits, top_ids, top_logits, top_lse, weights, True, out)
