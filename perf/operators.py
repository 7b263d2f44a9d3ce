"""The operators of a decoder that reads an encoder's states, as they are timed: the embedding lookup with its
gradient, the per-head norms of queries and keys with the position rotation, and cross attention.

A case is one pass of one operator:
  embed : y = scale * table[id] (a shard of the vocabulary's rows; zero rows for ids of other shards) and, with
          `backward`, the shard's dense fp32 gradient, zeros where no token points
  norm  : RMS norm of every query and key head, a gain per column, rotation of the first `rot` columns by the token's
          position; with `backward` the gradients of queries, keys and gains
  cross : softmax(scale Q K^T over the keys that count) V, several query heads to a key head; a query that no key
          counts for gives zeros; with `backward` the gradients of Q, K and V
"""
import math

import torch

own = False

DEV = "cuda:0"
_EPS = 1e-6


def _embed(name, tokens, hidden, rows, dtype="bf16", shards=1, shard=0, scale=1.0, pad=False, backward=True):
    return dict(name=name, kind="embed", tokens=tokens, hidden=hidden, rows=rows, dtype=dtype, shards=shards, shard=shard,
                scale=scale, pad=pad, backward=backward)


def _norm(name, batch, q_len, k_len, q_heads, k_heads, head_dim, rot, dtype="bf16", pairs=False, packed=True, max_pos=4096,
          backward=True):
    return dict(name=name, kind="norm", batch=batch, q_len=q_len, k_len=k_len, q_heads=q_heads, k_heads=k_heads,
                head_dim=head_dim, rot=rot, dtype=dtype, pairs=pairs, packed=packed, max_pos=max_pos, backward=backward)


def _cross(name, batch, q_len, k_len, q_heads, k_heads, head_dim, dtype="bf16", ragged=False, holes=False, backward=True):
    return dict(name=name, kind="cross", batch=batch, q_len=q_len, k_len=k_len, q_heads=q_heads, k_heads=k_heads,
                head_dim=head_dim, dtype=dtype, ragged=ragged, holes=holes, backward=backward)


def listed():
    return [
        # one decoding step of 16 sequences: a lookup that is all latency
        _embed("embed_step", 16, 5120, 32000, backward=False, scale=math.sqrt(5120)),
        # full precision at the repository's small configuration (C1): parity runs
        _embed("embed_f32_small", 257, 256, 1001, dtype="f32"),
        # C2's tokens: a training step's lookup and gradient, whole vocabulary on one GPU
        _embed("embed_train", 8192, 2048, 32768, scale=math.sqrt(2048)),
        # a rank's half of a large vocabulary, odd counts, a quarter of the tokens padding, which has no gradient
        _embed("embed_shard_large", 16385, 4096, 64013, shards=2, shard=1, pad=True),
        # one decoding step of 64 sequences at positions of their own
        _norm("norm_step", 64, 1, 1, 40, 8, 128, 128, max_pos=32768, backward=False),
        # a full-precision block with a partial rotation by neighbouring columns, odd length
        _norm("norm_f32_odd", 3, 1001, 1001, 16, 16, 64, 32, dtype="f32", pairs=True),
        # C3's tokens, unsharded heads in four groups to a key head, read from the packed projection
        _norm("norm_train", 2, 2048, 2048, 32, 8, 128, 128),
        # one query against a short utterance's states: all latency
        _cross("cross_step_small", 1, 1, 1500, 16, 16, 64, backward=False),
        # one decoding step of 16 sequences over long, ragged encoder states, five query heads to a key head
        _cross("cross_step_long", 16, 1, 8192, 40, 8, 128, ragged=True, backward=False),
        # full precision, small and odd, with holes in the keys and a sample without any
        _cross("cross_f32_holes", 3, 257, 333, 8, 4, 64, dtype="f32", holes=True),
        # C2's tokens against ragged encoder states of another length
        _cross("cross_train", 4, 2048, 1501, 16, 16, 128, ragged=True),
        # C4's length on both sides, grouped heads, two samples: matrix work
        _cross("cross_train_large", 2, 4096, 4096, 32, 8, 128),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14))


_MOST = None


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi):
    return min(hi, max(lo, round(_log_uniform(rng, lo, hi))))


def _drawn(rng):
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    kind = rng.random()
    if kind < 0.25:
        shards = rng.choice((1, 1, 2, 4))
        return _embed("", _size(rng, 1, 32768), 8 * _size(rng, 8, 1024), _size(rng, 100, 131072), dtype, shards,
                      rng.randrange(shards), rng.choice((1.0, 0.5, 32.0)), rng.random() < 0.4, rng.random() < 0.75)
    head_dim = rng.choice((64, 128, 128))
    k_heads = rng.choice((1, 2, 4, 8, 16))
    q_heads = min(k_heads * rng.choice((1, 1, 2, 3, 4, 5, 8)), 64 // k_heads * k_heads)
    if kind < 0.5:
        head_dim = rng.choice((32, 64, 80, 96, 128, 128, 256))
        alike = rng.random() < 0.7
        q_len = 1 if rng.random() < 0.25 else _size(rng, 2, 8192)
        k_len = q_len if alike else _size(rng, 1, 8192)
        rot = 16 * rng.randrange(0, head_dim // 16 + 1) if rng.random() < 0.4 else head_dim
        return _norm("", _size(rng, 1, 64), q_len, k_len, q_heads, k_heads, head_dim, rot, dtype, rng.random() < 0.3, alike,
                     rng.choice((4096, 32768, 131072)) + q_len + k_len, q_len > 1 and rng.random() < 0.75)
    if kind < 0.7:
        return _cross("", _size(rng, 1, 64), rng.choice((1, 1, 1, 2, 5)), _size(rng, 1, 65536), q_heads, k_heads, head_dim, dtype,
                      rng.random() < 0.5, rng.random() < 0.2, False)
    return _cross("", _size(rng, 1, 8), _size(rng, 16, 8192), _size(rng, 1, 8192), q_heads, k_heads, head_dim, dtype,
                  rng.random() < 0.4, rng.random() < 0.2, rng.random() < 0.8)


def draw(rng):
    global _MOST
    if _MOST is None:
        _MOST = max(_cost(c) for c in listed())
    while True:
        c = _drawn(rng)
        del c["name"]
        scores = 0 if c["kind"] != "cross" else c["batch"] * c["q_heads"] * c["q_len"] * c["k_len"]
        if _cost(c) <= _MOST and scores <= 2 ** 30 and work(c)["bytes"] < 2 ** 32 and 3072 not in c.values():
            return c


# ---- inputs ---------------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, device=DEV, dtype=torch.float32).normal_(mean, std, generator=gen).to(dtype)


def _embed_inputs(c, seed):
    """Tokens follow the rank law of text (probability about 1 / rank), ranks spread over the ids at random; padding is id 0."""
    gen = _generator(seed)
    vocab = c["rows"] * c["shards"]
    rank = torch.exp(torch.rand(c["tokens"], device=DEV, generator=gen, dtype=torch.float64) * math.log(vocab)).long() - 1
    ids = torch.randperm(vocab, device=DEV, generator=gen)[rank.clamp(0, vocab - 1)]
    if c["pad"]:
        ids[torch.rand(c["tokens"], device=DEV, generator=gen) < 0.25] = c["shard"] * c["rows"]
    return dict(ids=ids, table=_normal(gen, (c["rows"], c["hidden"]), _dtype(c), 0.02),
                dy=_normal(gen, (c["tokens"], c["hidden"]), _dtype(c)) if c["backward"] else None)


def _norm_inputs(c, seed):
    gen = _generator(seed)
    b, hq, hk, dh, dt = c["batch"], c["q_heads"], c["k_heads"], c["head_dim"], _dtype(c)
    if c["packed"]:                                      # heads of the projection's output: [Q | K | V]
        qkv = _normal(gen, (b, c["q_len"], hq + 2 * hk, dh), dt)
        q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
    else:
        q, k = _normal(gen, (b, c["q_len"], hq, dh), dt), _normal(gen, (b, c["k_len"], hk, dh), dt)
    s = dict(q=q, k=k, gain_q=_normal(gen, (dh,), dt, 0.1, 1.0), gain_k=_normal(gen, (dh,), dt, 0.1, 1.0))
    half = c["rot"] // 2
    angle = torch.arange(c["max_pos"], device=DEV, dtype=torch.float64)[:, None] * (
        10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / max(half, 1)))
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    for side, n in (("q", c["q_len"]), ("k", c["k_len"])):
        first = torch.randint(0, c["max_pos"] - n + 1, (b, 1), device=DEV, generator=gen)
        s[side + "_pos"] = (first + torch.arange(n, device=DEV)).int()
    if c["packed"]:
        s["k_pos"] = s["q_pos"]
    if c["backward"]:
        s["dyq"], s["dyk"] = _normal(gen, tuple(q.shape), dt), _normal(gen, tuple(k.shape), dt)
    return s


def _cross_inputs(c, seed):
    gen = _generator(seed)
    b, hq, hk, dh, dt = c["batch"], c["q_heads"], c["k_heads"], c["head_dim"], _dtype(c)
    s = dict(q=_normal(gen, (b, c["q_len"], hq, dh), dt))
    kv = _normal(gen, (b, c["k_len"], 2 * hk, dh), dt)   # one projection of the encoder's states gives both
    s["k"], s["v"] = kv[:, :, :hk], kv[:, :, hk:]
    s["key_lens"] = s["key_mask"] = None
    if c["ragged"]:                                      # evenly from the whole length to half of it
        part = 1.0 - 0.5 * torch.randperm(b, device=DEV, generator=gen) / b
        s["key_lens"] = (part * c["k_len"]).round().int()
    if c["holes"]:
        s["key_mask"] = torch.rand(b, c["k_len"], device=DEV, generator=gen) < 0.8
        if b > 1:
            s["key_mask"][b - 1] = False
    if c["backward"]:
        s["do"] = _normal(gen, (b, c["q_len"], hq, dh), dt)
    return s


_INPUTS = {"embed": _embed_inputs, "norm": _norm_inputs, "cross": _cross_inputs}


def prepare(case, seed):
    state = dict(case=case, **_INPUTS[case["kind"]](case, seed))
    if own:
        from paper_2504_03662_amd import decoder_ops as ops
        if case["kind"] == "embed":
            first = case["shard"] * case["rows"]
            state["op"] = ops.DeviceEmbedding(case["rows"], case["hidden"], case["dtype"], case["scale"], first_row=first,
                                              pad_id=first if case["pad"] else -1)
        elif case["kind"] == "norm":
            state["op"] = ops.DeviceHeadNorm(case["head_dim"], case["rot"], case["dtype"], _EPS, pairs=case["pairs"])
        else:
            state["op"] = ops.DeviceCrossAttention(case["head_dim"], case["dtype"])
    return state


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return _RUN_OWN[state["case"]["kind"]](state) if own else _RUN_PLAIN[state["case"]["kind"]](state)


def _embed_own(s):
    y = s["op"].forward(s["table"], s["ids"])
    return dict(y=y, dtable=s["op"].backward(s["ids"], s["dy"])) if s["case"]["backward"] else dict(y=y)


def _norm_own(s):
    where = dict(cos=s["cos"], sin=s["sin"], q_pos=s["q_pos"], k_pos=s["k_pos"])
    q, k = s["op"].forward(s["q"], s["k"], s["gain_q"], s["gain_k"], **where)
    out = dict(q=q, k=k)
    if s["case"]["backward"]:
        out["dq"], out["dk"], out["dgain_q"], out["dgain_k"] = s["op"].backward(s["q"], s["k"], s["dyq"], s["dyk"], s["gain_q"],
                                                                               s["gain_k"], **where)
    return out


def _cross_own(s):
    keys = dict(key_lens=s["key_lens"], key_mask=s["key_mask"])
    if not s["case"]["backward"]:
        return dict(o=s["op"].forward(s["q"], s["k"], s["v"], want_lse=False, **keys)[0])
    o, lse = s["op"].forward(s["q"], s["k"], s["v"], **keys)
    dq, dk, dv = s["op"].backward(s["q"], s["k"], s["v"], o, lse, s["do"], **keys)
    return dict(o=o, dq=dq, dk=dk, dv=dv)


def _embed_plain(s):
    c = s["case"]
    first = c["shard"] * c["rows"]
    here = (s["ids"] >= first) & (s["ids"] < first + c["rows"])
    row = torch.where(here, s["ids"] - first, 0)
    y = s["table"][row].float() * c["scale"] * here[:, None]
    out = dict(y=y.to(s["table"].dtype))
    if c["backward"]:
        if c["pad"]:
            here = here & (s["ids"] != first)
        g = s["dy"].float() * (c["scale"] * here[:, None])
        out["dtable"] = torch.zeros(c["rows"], c["hidden"], device=DEV).index_add_(0, row, g)
    return out


def _turned(n, c, cos, sin, sign):
    """Columns (i, i + rot / 2), or (2 i, 2 i + 1) with `pairs`, turned by the position's i-th angle; sign -1: back."""
    rot = c["rot"]
    r = n[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["pairs"] else (r[..., :rot // 2], r[..., rot // 2:])
    x, y = a * cos - sign * b * sin, b * cos + sign * a * sin
    turned = torch.stack((x, y), dim=-1).flatten(-2) if c["pairs"] else torch.cat((x, y), dim=-1)
    return torch.cat((turned, n[..., rot:]), dim=-1)


def _norm_plain_side(s, x, gain, pos, dy):
    c = s["case"]
    cos, sin = s["cos"][pos.long()][:, :, None], s["sin"][pos.long()][:, :, None]
    f, g = x.float(), gain.float()
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + _EPS)
    u = f * r
    y = _turned(u * g, c, cos, sin, 1.0).to(x.dtype)
    if dy is None:
        return y, None, None
    dn = _turned(dy.float(), c, cos, sin, -1.0)
    du = dn * g
    dx = r * (du - u * (du * u).mean(-1, keepdim=True))
    return y, dx.to(x.dtype), (dn * u).sum((0, 1, 2))


def _norm_plain(s):
    q, dq, dgq = _norm_plain_side(s, s["q"], s["gain_q"], s["q_pos"], s.get("dyq"))
    k, dk, dgk = _norm_plain_side(s, s["k"], s["gain_k"], s["k_pos"], s.get("dyk"))
    return dict(q=q, k=k, dq=dq, dk=dk, dgain_q=dgq, dgain_k=dgk) if s["case"]["backward"] else dict(q=q, k=k)


def _counts(s):
    """Which keys count, [batch, keys], or None for all."""
    if s["key_lens"] is None:
        return s["key_mask"]
    here = torch.arange(s["k"].shape[1], device=DEV)[None] < s["key_lens"][:, None]
    return here if s["key_mask"] is None else here & s["key_mask"]


def _cross_plain(s):
    c = s["case"]
    b, hq, hk, dh = c["batch"], c["q_heads"], c["k_heads"], c["head_dim"]
    g, n, m = hq // hk, c["q_len"], c["k_len"]
    rows = lambda x: x.float().reshape(b, n, hk, g, dh).permute(0, 2, 1, 3, 4).reshape(b * hk, n * g, dh)
    cols = lambda x: x.float().permute(0, 2, 1, 3).reshape(b * hk, m, dh)
    back = lambda x, t: x.reshape(b, hk, n, g, dh).permute(0, 2, 1, 3, 4).reshape(b, n, hq, dh).to(t)
    back_k = lambda x, t: x.reshape(b, hk, m, dh).permute(0, 2, 1, 3).to(t)
    q, k, v, scale = rows(s["q"]), cols(s["k"]), cols(s["v"]), 1.0 / math.sqrt(dh)
    p = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    counts = _counts(s)
    if counts is not None:
        none = ~counts[:, None, :].expand(b, hk, m).reshape(b * hk, 1, m)
        p = p.masked_fill(none, -math.inf)
        v = v.masked_fill(none.transpose(1, 2), 0.0)
        k = k.masked_fill(none.transpose(1, 2), 0.0)
    top = p.amax(-1, keepdim=True)
    p = torch.exp(p - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v)
    out = dict(o=back(o, s["q"].dtype))
    if c["backward"]:
        do = rows(s["do"])
        dv = torch.matmul(p.transpose(1, 2).contiguous(), do)
        ds = p * (torch.matmul(do, v.transpose(1, 2).contiguous()) - (do * o).sum(-1, keepdim=True))
        out["dq"] = back(torch.matmul(ds, k) * scale, s["q"].dtype)
        out["dk"] = back_k(torch.matmul(ds.transpose(1, 2).contiguous(), q) * scale, s["k"].dtype)
        out["dv"] = back_k(dv, s["v"].dtype)
    return out


_RUN_OWN = {"embed": _embed_own, "norm": _norm_own, "cross": _cross_own}
_RUN_PLAIN = {"embed": _embed_plain, "norm": _norm_plain, "cross": _cross_plain}


# ---- what a pass cannot do without ----------------------------------------------------------------

def _distinct(c):
    """Expected number of different rows of this shard that the tokens point to."""
    vocab, t = c["rows"] * c["shards"], c["tokens"] * (0.75 if c["pad"] else 1.0)
    # rank r has probability log(1 + 1 / r) / log(vocab); all ranks up to 1000, beyond that by the integral's mid-points
    ranks = [(r, 1.0) for r in range(1, min(vocab, 1001))]
    lo = 1001.0
    while lo < vocab:
        hi = min(lo * 1.05, float(vocab))
        ranks.append(((lo + hi) / 2, hi - lo))
        lo = hi
    total = math.log(vocab) if vocab > 1 else 1.0
    found = sum(n * -math.expm1(t * math.log1p(-min(0.999999, math.log1p(1 / r) / total))) for r, n in ranks)
    return min(found / c["shards"] + (1 if c["pad"] else 0), c["rows"], c["tokens"])


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["kind"] == "embed":
        t, h = c["tokens"], c["hidden"]
        back = c["backward"]
        live = 0.75 * t / c["shards"] if c["pad"] else t / c["shards"]           # tokens with a gradient
        n = 8 * t + (t + _distinct(c)) * h * e + (live * h * e + 4 * c["rows"] * h if back else 0)
        return {"bytes": int(n), "flops": int(t * h + (2 * live * h if back else 0))}
    if c["kind"] == "norm":
        b, dh = c["batch"], c["head_dim"]
        heads = b * (c["q_len"] * c["q_heads"] + c["k_len"] * c["k_heads"])
        tokens = b * (c["q_len"] + (0 if c["packed"] else c["k_len"]))
        n = tokens * (4 + 4 * min(c["rot"], c["rot"] * c["max_pos"] // max(tokens, 1))) + 2 * dh * e
        back = c["backward"]
        return {"bytes": int(n + heads * dh * e * (4 if back else 2) + (8 * dh if back else 0)),
                "flops": int(heads * dh * (22 if back else 8))}
    b, hq, hk, dh = c["batch"], c["q_heads"], c["k_heads"], c["head_dim"]
    keys = b * c["k_len"]
    if c["ragged"]:
        keys = sum(round((1.0 - 0.5 * i / b) * c["k_len"]) for i in range(b))
    if c["holes"]:
        keys = int(0.8 * keys * (b - 1) / b if b > 1 else 0.8 * keys)
    q_bytes, kv_bytes = b * c["q_len"] * hq * dh * e, keys * 2 * hk * dh * e
    flops = 4 * c["q_len"] * keys * hq * dh
    if not c["backward"]:
        return {"bytes": int(2 * q_bytes + kv_bytes), "flops": int(flops)}
    return {"bytes": int(4 * q_bytes + kv_bytes + 2 * b * c["k_len"] * hk * dh * e), "flops": int(3.5 * flops)}


# ---- the answer in 64 bits, from the definitions --------------------------------------------------

def exact(case, seed):
    c, x = case, _INPUTS[case["kind"]](case, seed)
    if c["kind"] == "embed":
        return _embed_exact(c, x)
    if c["kind"] == "norm":
        q = _norm_exact(c, x["q"], x["gain_q"], x["cos"], x["sin"], x["q_pos"], x.get("dyq"))
        k = _norm_exact(c, x["k"], x["gain_k"], x["cos"], x["sin"], x["k_pos"], x.get("dyk"))
        out = dict(q=q[0], k=k[0])
        if c["backward"]:
            out.update(dq=q[1], dk=k[1], dgain_q=q[2], dgain_k=k[2])
        return out
    return _cross_exact(c, x)


def _embed_exact(c, x):
    """By the sorted ids: every run of equal ones is a difference of running sums' ends, per block of columns."""
    first, vocab = c["shard"] * c["rows"], c["rows"] * c["shards"]
    whole = torch.zeros(vocab + 1, c["hidden"], device=DEV, dtype=torch.float64)
    whole[first:first + c["rows"]] = x["table"].double()
    out = dict(y=whole[x["ids"]] * c["scale"])
    if c["backward"]:
        del whole
        g = torch.zeros(c["rows"], c["hidden"], device=DEV, dtype=torch.float64)
        ids = x["ids"].clone()
        ids[(ids < first) | (ids >= first + c["rows"])] = -1
        if c["pad"]:
            ids[ids == first] = -1
        order = torch.argsort(ids, stable=True)
        order = order[ids[order] >= 0]
        if order.numel():
            row, count = torch.unique_consecutive(ids[order], return_counts=True)
            g[row - first] = torch.segment_reduce(x["dy"][order].double() * c["scale"], "sum", lengths=count, axis=0)
        out["dtable"] = g
    return out


def _norm_exact(c, x, gain, cos, sin, pos, dy):
    """The columns as complex numbers, and the gradients by automatic differentiation."""
    half = c["rot"] // 2
    x, gain = x.double().detach().requires_grad_(), gain.double().detach().requires_grad_()
    n = gain * x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + _EPS)
    turn = torch.complex(cos.double(), sin.double())[pos.long()].unsqueeze(2)
    at = torch.arange(c["rot"], device=DEV)
    re, im = (at[0::2], at[1::2]) if c["pairs"] else (at[:half], at[half:])
    z = torch.complex(n[..., re], n[..., im]) * turn
    y = n.clone()
    y[..., re], y[..., im] = z.real, z.imag
    if dy is None:
        return y.detach(), None, None
    dx, dgain = torch.autograd.grad(y, (x, gain), dy.double())
    return y.detach(), dx, dgain


def _cross_exact(c, x):
    """Sample by sample and head by head, over the keys that count alone."""
    b, g, dh = c["batch"], c["q_heads"] // c["k_heads"], c["head_dim"]
    counts = _counts(x)
    zeros = lambda t: torch.zeros(t.shape, device=DEV, dtype=torch.float64)
    o, dq, dk, dv = zeros(x["q"]), zeros(x["q"]), zeros(x["k"]), zeros(x["v"])
    for i in range(b):
        at = torch.arange(c["k_len"], device=DEV) if counts is None else counts[i].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        for h in range(c["q_heads"]):
            q, k, v = x["q"][i, :, h].double(), x["k"][i, at, h // g].double(), x["v"][i, at, h // g].double()
            p = torch.softmax(q @ k.t().contiguous() / math.sqrt(dh), dim=-1)
            o[i, :, h] = p @ v
            if c["backward"]:
                do = x["do"][i, :, h].double()
                dp = do @ v.t().contiguous()
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(dh)
                dq[i, :, h] = ds @ k
                dk[i, at, h // g] += ds.t().contiguous() @ q
                dv[i, at, h // g] += p.t().contiguous() @ do
    return dict(o=o, dq=dq, dk=dk, dv=dv) if c["backward"] else dict(o=o)
