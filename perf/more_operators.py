"""What a decoder learns from, as it is timed: losses of its logits together with the logits' gradient.

A case is one pass of one operator over logits z [rows, vocab] (p = softmax(scale z), logp = log p of the row's token):
  token      : cross entropy -w logp with its gradient, or `score`: the tokens' log probabilities and log sums alone
  logp       : log probabilities over one shard of the vocabulary, and the gradient that given dlogp and the whole
               vocabulary's log sums make of them
  policy     : w (-min(r A, clip(r) A) + kl (exp(d) - d - 1)), r = exp(logp - old), d = ref - logp, with its gradient
  preference : pairs of sequences; x = beta (sum of w (logp - ref) over the chosen one - the same over the rejected one)
               - margin, loss -(1 - s) log sigmoid(x) - s log sigmoid(-x), with its gradient
  distill    : sum of q log(q / p) over a teacher's top entries, q their softmax or, with `rest`, their probabilities
               by the teacher's own log sum, the remaining tokens then being one more outcome; with its gradient
"""
import math

import torch

own = False

DEV = "cuda:0"
_IGNORE = -1


def _token(name, rows, vocab, dtype="bf16", scale=1.0, ignored=0.0, pad=0, score=False):
    return dict(name=name, kind="token", rows=rows, vocab=vocab, dtype=dtype, scale=scale, ignored=ignored, pad=pad, score=score)


def _logp(name, rows, vocab, shards, shard, dtype="bf16", scale=1.0, ignored=0.0, pad=0):
    return dict(name=name, kind="logp", rows=rows, vocab=vocab, shards=shards, shard=shard, dtype=dtype, scale=scale, ignored=ignored,
                pad=pad)


def _policy(name, rows, vocab, dtype="bf16", scale=1.0, ignored=0.0, pad=0, low=0.2, high=0.2, kl=0.05):
    return dict(name=name, kind="policy", rows=rows, vocab=vocab, dtype=dtype, scale=scale, ignored=ignored, pad=pad, low=low, high=high,
                kl=kl)


def _preference(name, pairs, rows, vocab, dtype="bf16", ignored=0.25, pad=0, beta=0.1, margin=0.0, smoothing=0.0, reference=True):
    return dict(name=name, kind="preference", pairs=pairs, rows=rows, vocab=vocab, dtype=dtype, scale=1.0, ignored=ignored, pad=pad,
                beta=beta, margin=margin, smoothing=smoothing, reference=reference)


def _distill(name, rows, vocab, top, dtype="bf16", scale=1.0, ignored=0.0, pad=0, rest=False):
    return dict(name=name, kind="distill", rows=rows, vocab=vocab, top=top, dtype=dtype, scale=scale, ignored=ignored, pad=pad, rest=rest)


def listed():
    return [
        # a step of 16 sequences: the log probabilities of the tokens just drawn, all latency
        _token("token_score_step", 16, 32000, score=True),
        # full precision at the size of the repository's small configuration (C1), odd counts, some tokens padding
        _token("token_f32_odd", 257, 1001, dtype="f32", ignored=0.2),
        # C2's tokens: a training step's loss and gradient, whole vocabulary on one GPU
        _token("token_train", 8192, 32768, ignored=0.05),
        # a rank's half of a large vocabulary of an odd size, so that rows begin at any element
        _logp("logp_shard", 4096, 64013, 2, 1),
        # one small minibatch of sampled tokens
        _policy("policy_small", 64, 32000),
        # full precision, odd counts, a sampling temperature, a wider upper border
        _policy("policy_f32_odd", 1001, 5003, dtype="f32", scale=1.25, ignored=0.3, high=0.28),
        # 8192 sampled tokens and their prompts, odd vocabulary
        _policy("policy_train", 8192, 50001, ignored=0.25),
        # two short pairs in full precision: the gradient of a few rows, launches in a chain
        _preference("preference_small", 2, 131, 1001, dtype="f32"),
        # 8 pairs of ragged sequences packed into C2's tokens, prompts not counted
        _preference("preference_train", 8, 8192, 32768, smoothing=0.1),
        # a few tokens against a teacher's 16 largest logits
        _distill("distill_small", 32, 32000, 16),
        # C3's tokens against 64 stored logits of a teacher, vocabulary padded to a multiple of the matrix tile
        _distill("distill_train", 4096, 32003, 64, pad=61, ignored=0.1),
        # a large vocabulary, 256 stored logits and their teacher's log sums, temperature 2
        _distill("distill_rest_large", 2048, 131072, 256, scale=0.5, rest=True),
    ]


_MOST = None


def _size(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _drawn(rng):
    kind = rng.choice(("token", "logp", "policy", "preference", "distill"))
    common = dict(dtype="f32" if rng.random() < 0.3 else "bf16", ignored=rng.choice((0.0, 0.1, 0.3, 0.6)), pad=rng.choice((0, 0, 0, 1, 6, 56)))
    rows, vocab = _size(rng, 1, 16384), _size(rng, 100, 262144)
    if rng.random() < 0.4:
        vocab = max(128, vocab // 64 * 64)
    scale = rng.choice((1.0, 1.0, 0.5, 0.7, 2.0))
    if kind == "token":
        return _token("", rows, vocab, scale=scale, score=rng.random() < 0.3, **common)
    if kind == "logp":
        shards = rng.choice((2, 3, 4, 8))
        return _logp("", rows, vocab, shards, rng.randrange(shards), scale=scale, **common)
    if kind == "policy":
        return _policy("", rows, vocab, scale=scale, low=rng.choice((0.1, 0.2)), high=rng.choice((0.1, 0.2, 0.28)),
                       kl=rng.choice((0.0, 0.01, 0.1)), **common)
    if kind == "preference":
        return _preference("", min(_size(rng, 1, 64), max(1, rows // 4)), max(rows, 4), vocab, beta=rng.choice((0.05, 0.1, 0.5)),
                           margin=rng.choice((0.0, 0.0, 0.5)), smoothing=rng.choice((0.0, 0.1)), reference=rng.random() < 0.8, **common)
    return _distill("", rows, vocab, min(_size(rng, 1, 512), vocab), scale=scale, rest=rng.random() < 0.5, **common)


def draw(rng):
    global _MOST
    if _MOST is None:
        _MOST = max(work(c)["bytes"] for c in listed())
    while True:
        c = _drawn(rng)
        del c["name"]
        if work(c)["bytes"] <= _MOST:
            return c


# ---- inputs ---------------------------------------------------------------------------------------

def _chunks(n, vocab):
    step = max(1, (1 << 27) // vocab)
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


def _inputs(c, seed):
    """Logits as a trained model has them: one token of a row, more often than not the one that comes, stands out."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, v = c["rows"], c["vocab"]
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    uniform = lambda *shape: torch.rand(shape, device=DEV, generator=gen)
    normal = lambda *shape: torch.randn(shape, device=DEV, generator=gen)
    whole = torch.empty(n, v + c["pad"], device=DEV, dtype=dtype)
    for at in _chunks(n, v):
        whole[at] = (2.0 * normal(whole[at].shape[0], v + c["pad"])).to(dtype)
    z = whole[:, :v]
    first = c.get("shard", 0) * v
    ids = torch.randint(0, v * c.get("shards", 1), (n,), device=DEV, generator=gen)
    peak = torch.where(uniform(n) < 0.6, (ids - first).clamp(0, v - 1), torch.randint(0, v, (n,), device=DEV, generator=gen))
    row = torch.arange(n, device=DEV)
    z[row, peak] = (z[row, peak].float() + 4.0 + 10.0 * uniform(n)).to(dtype)
    counts = uniform(n) >= c["ignored"]
    s = dict(logits=z, ids=ids)
    if c["kind"] in ("token", "logp"):
        s["ids"] = torch.where(counts, ids, _IGNORE)
    if c["kind"] in ("token", "policy", "distill"):
        s["weights"] = counts / counts.sum().clamp(min=1)
    if c["kind"] == "distill":
        s.update(_teacher(c, z, gen))
        return s
    lse = torch.cat([torch.logsumexp(z[at].float() * c["scale"], 1) for at in _chunks(n, v)])
    if c["kind"] == "logp":                              # the other shards hold about as much as this one
        s["lse_all"] = lse + math.log(c["shards"]) + 0.1 * normal(n)
        s["dlogp"] = torch.where(counts, normal(n) / n, 0.0)
    if c["kind"] in ("policy", "preference"):
        logp = z[row, ids].float() * c["scale"] - lse
    if c["kind"] == "policy":
        # how far the policy has moved since it sampled; on which side of a border a ratio lies is not left to a rounding
        ratio = 0.2 * normal(n)
        for border in (math.log1p(c["high"]), math.log1p(-c["low"])):
            ratio = torch.where((ratio - border).abs() < 1e-3, border + torch.where(ratio < border, -1e-3, 1e-3), ratio)
        s["old"] = logp - ratio
        s["ref"] = logp + 0.3 * normal(n) if c["kl"] else None
        one = normal(n // 64 + 1)                        # an answer's tokens share its advantage; a group alike has none
        s["adv"] = torch.where(one.abs() < 0.1, 0.0, one)[row // 64]
    if c["kind"] == "preference":
        s["ref"] = logp + 0.1 * normal(n) if c["reference"] else None
        cut = torch.randperm(max(n - n // 64, 2 * c["pairs"]), device=DEV, generator=gen)[:2 * c["pairs"]].sort().values + 1
        s["starts"] = torch.cat([torch.zeros(1, device=DEV, dtype=torch.long), cut]).int()
        s["weights"] = counts.float()
        s["pair_weights"] = torch.full((c["pairs"],), 1.0 / c["pairs"], device=DEV)
        if not c["reference"]:                           # mean log probabilities instead: sequences of any length compare
            seq = torch.searchsorted(cut, row, right=True)
            total = torch.zeros(2 * c["pairs"] + 1, device=DEV).index_add_(0, seq, s["weights"])
            s["weights"] = s["weights"] / total[seq].clamp(min=1.0)
    return s


def _teacher(c, z, gen):
    """The largest logits of a teacher that sees what the student sees, with noise of its own, and its log sums."""
    top = {"top_ids": [], "top_logits": [], "top_lse": []}
    for at in _chunks(c["rows"], c["vocab"]):
        t = z[at].float() + 0.5 * torch.randn(z[at].shape, device=DEV, generator=gen)
        best = t.topk(c["top"], dim=1)
        top["top_ids"].append(best.indices.int())
        top["top_logits"].append(best.values if c["rest"] else best.values.to(z.dtype))
        top["top_lse"].append(torch.logsumexp(t * c["scale"], 1))
    top = {k: torch.cat(x) for k, x in top.items()}
    if not c["rest"]:
        top["top_lse"] = None
    return top


def prepare(case, seed):
    c = case
    state = dict(case=c, **_inputs(c, seed))
    if own:
        from paper_2504_03662_amd import loss_ops as ops
        if c["kind"] in ("token", "logp"):
            state["op"] = ops.DeviceTokenLoss(c["vocab"], c["dtype"], scale=c["scale"], ignore_id=_IGNORE,
                                              first_id=c.get("shard", 0) * c["vocab"], whole_vocab=c.get("shards", 1) * c["vocab"])
        elif c["kind"] == "policy":
            state["op"] = ops.DevicePolicyLoss(c["vocab"], c["dtype"], clip_low=c["low"], clip_high=c["high"], kl=c["kl"], scale=c["scale"])
        elif c["kind"] == "preference":
            state["op"] = ops.DevicePreferenceLoss(c["vocab"], c["dtype"], beta=c["beta"], margin=c["margin"], smoothing=c["smoothing"])
        else:
            state["op"] = ops.DeviceDistillation(c["vocab"], c["dtype"], scale=c["scale"])
    return state


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["case"]["kind"]](state)


def _token_own(s):
    if s["case"]["score"]:
        logp, lse = s["op"].logp(s["logits"], s["ids"])
        return dict(logp=logp, lse=lse)
    loss, dlogits = s["op"].forward_backward(s["logits"], s["ids"], s["weights"])
    return dict(loss=loss, dlogits=dlogits)


def _logp_own(s):
    logp, lse = s["op"].logp(s["logits"], s["ids"])
    return dict(logp=logp, lse=lse, dlogits=s["op"].logp_backward(s["logits"], s["ids"], s["lse_all"], s["dlogp"]))


def _policy_own(s):
    loss, logp, dlogits = s["op"].forward_backward(s["logits"], s["ids"], s["old"], s["adv"], ref_logp=s["ref"], weights=s["weights"])
    return dict(loss=loss, logp=logp, dlogits=dlogits)


def _preference_own(s):
    loss, rewards, dlogits = s["op"].forward_backward(s["logits"], s["ids"], s["starts"], ref_logp=s["ref"], weights=s["weights"],
                                                      pair_weights=s["pair_weights"])
    return dict(loss=loss, rewards=rewards, dlogits=dlogits)


def _distill_own(s):
    loss, dlogits = s["op"].forward_backward(s["logits"], s["top_ids"], s["top_logits"], top_lse=s["top_lse"], weights=s["weights"])
    return dict(loss=loss, dlogits=dlogits)


def _scaled(s):
    """(scale z less its row's maximum, that maximum, the sum of the exponentials).  The sum, its logarithm and what is taken from
    it are in 64 bits: losses are small differences of them, rewards sums over many tokens."""
    x = s["logits"].float() * s["case"]["scale"]
    top = x.amax(1, keepdim=True)
    x = x - top
    return x, top, x.exp().sum(1, keepdim=True, dtype=torch.float64)


def _picked(s, x, total):
    return torch.gather(x, 1, s["ids"][:, None])[:, 0] - total[:, 0].log()


def _gradient(s, x, total, g):
    """g dlogp / dz, rows with g = 0 left out"""
    c = s["case"]
    d = x.exp() * (-c["scale"] * g[:, None] / total.float())
    first = c.get("shard", 0) * c["vocab"]
    here = (s["ids"] >= first) & (s["ids"] < first + c["vocab"])
    at = torch.where(here, s["ids"] - first, 0)[:, None]
    d.scatter_add_(1, at, (c["scale"] * g * here)[:, None])
    return torch.where(g[:, None] == 0, 0.0, d).to(s["logits"].dtype)


def _token_plain(s):
    x, top, total = _scaled(s)
    counts = s["ids"] != _IGNORE
    s = dict(s, ids=torch.where(counts, s["ids"], 0))
    logp = torch.where(counts, _picked(s, x, total), 0.0)
    if s["case"]["score"]:
        return dict(logp=logp.float(), lse=torch.where(counts, (total.log() + top)[:, 0], 0.0).float())
    w = torch.where(counts, s["weights"], 0.0)
    return dict(loss=(-w * logp).float(), dlogits=_gradient(s, x, total, -w))


def _logp_plain(s):
    c, first = s["case"], s["case"]["shard"] * s["case"]["vocab"]
    x, top, total = _scaled(s)
    counts = s["ids"] != _IGNORE
    here = (s["ids"] >= first) & (s["ids"] < first + c["vocab"])
    lse = (total.log() + top)[:, 0]
    picked = torch.gather(x, 1, torch.where(here, s["ids"] - first, 0)[:, None])[:, 0] - total.log()[:, 0]
    logp = torch.where(here, picked, -lse)
    d = _gradient(s, x + (top - s["lse_all"][:, None]), torch.ones_like(total), torch.where(counts, s["dlogp"], 0.0))
    return dict(logp=torch.where(counts, logp, 0.0).float(), lse=torch.where(counts, lse, 0.0).float(), dlogits=d)


def _policy_plain(s):
    c = s["case"]
    x, top, total = _scaled(s)
    logp = _picked(s, x, total)
    r = torch.exp(logp - s["old"])
    plain, cut = r * s["adv"], r.clamp(1.0 - c["low"], 1.0 + c["high"]) * s["adv"]
    loss, g = -torch.minimum(plain, cut), torch.where(plain <= cut, -plain, 0.0)
    if s["ref"] is not None:
        d = s["ref"] - logp
        loss, g = loss + c["kl"] * (d.exp() - d - 1.0), g + c["kl"] * (1.0 - d.exp())
    return dict(loss=(s["weights"] * loss).float(), logp=torch.where(s["weights"] != 0, logp, 0.0).float(),
                dlogits=_gradient(s, x, total, (s["weights"] * g).float()))


def _preference_plain(s):
    c, n = s["case"], s["case"]["rows"]
    x, top, total = _scaled(s)
    logp = _picked(s, x, total)
    ends = s["starts"][1:].long()
    seq = torch.searchsorted(ends, torch.arange(n, device=DEV), right=True)              # 2 pairs: behind the last one
    gain = s["weights"].double() * (logp if s["ref"] is None else logp - s["ref"].double())
    sums = torch.zeros(2 * c["pairs"] + 1, device=DEV, dtype=torch.float64).index_add_(0, seq, gain)[:-1]
    chosen, rejected = sums[0::2], sums[1::2]
    at = (c["beta"] * (chosen - rejected) - c["margin"]).float()
    low = torch.log1p(torch.exp(-at.abs()))                                              # -log sigmoid(|x|)
    loss = (1.0 - c["smoothing"]) * (low + (-at).clamp(min=0.0)) + c["smoothing"] * (low + at.clamp(min=0.0))
    slope = s["pair_weights"] * (c["smoothing"] - 1.0 / (1.0 + torch.exp(at))) * c["beta"]
    g = torch.cat([torch.stack((slope, -slope), 1).flatten(), torch.zeros(1, device=DEV)])[seq] * s["weights"]
    return dict(loss=s["pair_weights"] * loss, rewards=(c["beta"] * sums).float(), dlogits=_gradient(s, x, total, g))


def _distill_plain(s):
    c = s["case"]
    x, top, total = _scaled(s)
    at, t = s["top_ids"].long(), s["top_logits"].double() * c["scale"]
    if s["top_lse"] is None:
        logq = t - t.amax(1, keepdim=True)
        logq = logq - logq.exp().sum(1, keepdim=True).log()
    else:
        logq = t - s["top_lse"].double()[:, None]
    q, log_total = logq.exp(), total.log()
    logp = torch.gather(x, 1, at) - log_total
    loss = (q * (logq - logp)).sum(1)
    p = x.exp() / total.float()
    teacher = torch.zeros_like(x).scatter_add_(1, at, q.float())
    mass = q.sum(1)
    if s["top_lse"] is not None:
        r = (1.0 - mass).clamp(min=0.0)
        y = x.scatter(1, at, -math.inf)
        best = y.amax(1, keepdim=True)
        some = best[:, 0] > -math.inf
        r = torch.where(some, r, 0.0)
        e = torch.where(some[:, None], torch.exp(y - best), 0.0)
        tail = e.sum(1, keepdim=True, dtype=torch.float64)
        others = torch.where(r > 0, r * (torch.where(r > 0, r, 1.0).log() - (best + tail.log() - log_total)[:, 0]), 0.0)
        loss, mass = loss + others, mass + r
        teacher += torch.where(some[:, None], r.float()[:, None] * e / tail.float(), 0.0)
    w = s["weights"]
    d = (c["scale"] * w)[:, None] * (mass.float()[:, None] * p - teacher)
    return dict(loss=(w * loss).float(), dlogits=torch.where(w[:, None] == 0, 0.0, d).to(s["logits"].dtype))


_RUN_OWN = {"token": _token_own, "logp": _logp_own, "policy": _policy_own, "preference": _preference_own, "distill": _distill_own}
_RUN_PLAIN = {"token": _token_plain, "logp": _logp_plain, "policy": _policy_plain, "preference": _preference_plain,
              "distill": _distill_plain}


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    """Logits of the rows that count in, a gradient of every row out; an exponential, a few products and sums to an element"""
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    n, v, live = c["rows"], c["vocab"], 1.0 - c["ignored"]
    back = not c.get("score", False)
    small = {"token": 16, "logp": 28, "policy": 32, "preference": 16, "distill": 8}[c["kind"]] * n
    if c["kind"] == "distill":
        small += n * c["top"] * (8 if c["rest"] else 4 + e)
    return {"bytes": int(live * n * v * e + (n * v * e if back else 0) + small), "flops": int(live * n * v * (7 if back else 4))}


# ---- the answer in 64 bits, from the definitions --------------------------------------------------

def exact(case, seed):
    c, x = case, _inputs(case, seed)
    n, v, scale = c["rows"], c["vocab"], c["scale"]
    if c["kind"] == "preference":
        return _preference_exact(c, x)
    parts = []
    for at in _chunks(n, 4 * v):
        y = {k: t[at] if torch.is_tensor(t) and t.shape[0] == n else t for k, t in x.items()}
        z = y["logits"].double().requires_grad_()
        parts.append(_EXACT[c["kind"]](c, y, z, scale * z))
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _token_exact(c, y, z, a):
    on = y["ids"] != _IGNORE
    row = torch.arange(len(on), device=DEV)[on]
    logp = torch.zeros(len(on), device=DEV, dtype=torch.float64)
    logp[on] = torch.log_softmax(a, 1)[row, y["ids"][on]]
    if c["score"]:
        return dict(logp=logp.detach(), lse=torch.logsumexp(a, 1).detach() * on)
    loss = -y["weights"].double() * logp
    return dict(loss=loss.detach(), dlogits=torch.autograd.grad(loss.sum(), z)[0])


def _logp_exact(c, y, z, a):
    ids, first = y["ids"], c["shard"] * c["vocab"]
    on = ids != _IGNORE
    mine = (ids >= first) & (ids < first + c["vocab"])
    row = torch.arange(len(on), device=DEV)
    a = a.detach()
    lse = torch.logsumexp(a, 1)
    logp = -lse
    logp[mine] += a[row[mine], ids[mine] - first]
    g = (c["scale"] * y["dlogp"].double() * on)[:, None]
    d = -g * torch.exp(a - y["lse_all"].double()[:, None])
    d[row[mine], ids[mine] - first] += g[mine, 0]
    return dict(logp=logp * on, lse=lse * on, dlogits=d)


def _policy_exact(c, y, z, a):
    w, adv = y["weights"].double(), y["adv"].double()
    logp = torch.log_softmax(a, 1).gather(1, y["ids"][:, None])[:, 0]
    gain = logp - y["old"].double()
    over = torch.where(adv > 0, gain.detach() > math.log1p(c["high"]), gain.detach() < math.log1p(-c["low"])) & (adv != 0)
    border = torch.where(adv > 0, 1.0 + c["high"], 1.0 - c["low"]).double()
    loss = -adv * torch.where(over, border, torch.exp(gain))
    if y["ref"] is not None:
        d = y["ref"].double() - logp
        loss = loss + c["kl"] * (torch.expm1(d) - d)
    loss = w * loss
    return dict(loss=loss.detach(), logp=(logp * (w != 0)).detach(), dlogits=torch.autograd.grad(loss.sum(), z)[0])


def _preference_exact(c, x):
    """Sequence by sequence"""
    z, ids = x["logits"], x["ids"]
    parts = _chunks(c["rows"], 4 * c["vocab"])
    logp = torch.cat([torch.log_softmax(z[at].double(), 1).gather(1, ids[at][:, None])[:, 0] for at in parts]).requires_grad_()
    ends = x["starts"].tolist()
    w = x["weights"].double()
    gain = w * (logp if x["ref"] is None else logp - x["ref"].double())
    rewards = c["beta"] * torch.stack([gain[a:b].sum() for a, b in zip(ends, ends[1:])])
    at = rewards[0::2] - rewards[1::2] - c["margin"]
    s = c["smoothing"]
    loss = -x["pair_weights"].double() * ((1 - s) * torch.nn.functional.logsigmoid(at) + s * torch.nn.functional.logsigmoid(-at))
    g, = torch.autograd.grad(loss.sum(), logp)
    d = torch.empty(z.shape, device=DEV, dtype=torch.float64)
    for at in parts:
        d[at] = torch.softmax(z[at].double(), 1) * -g[at][:, None]
    d[torch.arange(c["rows"], device=DEV), ids] += g
    return dict(loss=loss.detach(), rewards=rewards.detach(), dlogits=d)


def _distill_exact(c, y, z, a):
    """Over the outcomes: the teacher's entries and, with its log sums, all other tokens as one"""
    t = c["scale"] * y["top_logits"].double()
    at = y["top_ids"].long()
    logp = torch.log_softmax(a, 1)
    if y["top_lse"] is None:
        logq, logp = torch.log_softmax(t, 1), logp.gather(1, at)
    else:
        logq = t - y["top_lse"].double()[:, None]
        r = (1.0 - logq.exp().sum(1, keepdim=True)).clamp(min=0.0)
        others = torch.ones(a.shape, device=DEV, dtype=torch.bool).scatter_(1, at, False)
        tail = torch.logsumexp(logp.masked_fill(~others, -math.inf), 1, keepdim=True)
        logp, logq = logp.gather(1, at), logq
        if c["top"] < c["vocab"]:
            logp, logq = torch.cat([logp, tail], 1), torch.cat([logq, r.log()], 1)
    q = logq.exp()
    terms = torch.where(q > 0, q * (torch.where(q > 0, logq, 0.0) - logp), 0.0)
    loss = y["weights"].double() * terms.sum(1)
    return dict(loss=loss.detach(), dlogits=torch.autograd.grad(loss.sum(), z)[0])


_EXACT = {"token": _token_exact, "logp": _logp_exact, "policy": _policy_exact, "distill": _distill_exact}
