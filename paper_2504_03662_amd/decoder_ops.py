"""The operators around a block of a decoder that reads an encoder's states, on torch tensors: the token embedding and its
gradient, norms of queries and keys with the position rotation, and cross attention.  Like `runtime`, this is plumbing: torch
supplies device memory and the stream, shapes and types are checked here, and the library does all the compute.

Every call works on the current stream and returns without waiting.  An object holds sizes and scratch memory only, one piece of
scratch per stream and host thread, so that calls on different streams or of different threads (whose launches on one stream may
mix) do not meet, and none that a captured graph uses; tensors of another stream or thread are the caller's to order, as everywhere
in torch.  Outputs are new tensors unless `out`s are given."""
from __future__ import annotations

import threading

import torch

from . import binding as gx

_TYPES = {"bf16": (gx.GX_BF16, torch.bfloat16), "f32": (gx.GX_F32, torch.float32)}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


class _Operator:
    """Type, device (which has to be the current one in calls) and scratch of an operator."""

    def __init__(self, dtype, device):
        gx.lib()                                   # fail loudly if the library is not built
        self.gtype, self.tdtype = _TYPES[dtype]
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.index = -1 if self.device.type == "cpu" else self.device.index
        # by host thread and stream (what a thread that has ended leaves is found by the next of its number)
        self._scratch = {}

    def _workspace(self, nbytes, stream):
        # A captured call has memory of its own, from the graph's pool: the graph keeps the address for as long as it lives, while
        # the memory that eager calls share is replaced when one needs more.
        capturing = torch.cuda.is_current_stream_capturing()
        key = threading.get_ident(), stream
        w = None if capturing else self._scratch.get(key)
        if w is None or w.numel() < nbytes:
            w = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            if not capturing:
                self._scratch[key] = w
        return w

    def _check(self, name, t, shape, dtype, contiguous=True):
        if t.dtype is dtype and t.get_device() == self.index and t.shape == shape and (not contiguous or t.is_contiguous()):
            return
        _need(t.dtype == dtype, f"{name}: {t.dtype}, not {dtype}")
        _need(t.get_device() == self.index, f"{name}: on {t.device}, not {self.device}")
        _need(t.shape == shape, f"{name}: shape {tuple(t.shape)}, not {tuple(shape)}")
        raise ValueError(f"{name}: not contiguous")

    def _heads(self, name, x):
        """The shape of a tensor of heads"""
        shape = x.shape
        if x.dtype is self.tdtype and x.get_device() == self.index and len(shape) == 4 and shape[3] == self.head_dim:
            return shape
        _need(len(shape) == 4 and shape[3] == self.head_dim, f"{name}: not [batch, tokens, heads, {self.head_dim}]")
        self._check(name, x, shape, self.tdtype, False)

    def _new(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _stream(self):
        # launches go to the current GPU, whatever stream they are given
        if torch._C._cuda_getDevice() != self.index:
            raise ValueError(f"{self.device} is not the current GPU")
        # the handle itself: a torch.cuda.Stream around it takes 2.8 us to make, a third of a small call
        return torch._C._cuda_getCurrentRawStream(self.index)


class DeviceEmbedding(_Operator):
    """Rows [first_row, first_row + rows) of a vocabulary: y = scale * table[ids - first_row], zeros for ids of other shards, and
    the table's gradient.  Tokens with `pad_id` have no gradient."""

    def __init__(self, rows, hidden, dtype="bf16", scale=1.0, first_row=0, pad_id=-1, device="cuda:0"):
        super().__init__(dtype, device)
        self.rows, self.hidden, self.scale, self.first_row, self.pad_id = rows, hidden, scale, first_row, pad_id

    def _cfg(self, ids, flags=0):
        _need(ids.dtype in (torch.int32, torch.int64), f"ids: {ids.dtype}, not int32 or int64")
        self._check("ids", ids, ids.shape, ids.dtype)
        return gx.EmbedCfg(ids.numel(), self.hidden, self.rows, self.gtype, ids.element_size(), flags, self.first_row, self.pad_id,
                           self.scale)

    def forward(self, table, ids, out=None):
        """table [rows, hidden], ids of any shape -> [*ids.shape, hidden]"""
        cfg, shape = self._cfg(ids), (*ids.shape, self.hidden)
        self._check("table", table, (self.rows, self.hidden), self.tdtype)
        if out is None:
            out = self._new(shape, self.tdtype)
        else:
            self._check("out", out, shape, self.tdtype)
        gx.embed_fwd(cfg, table, ids, out, self._stream())
        return out

    def backward(self, ids, dy, out=None, accumulate=False):
        """dy [*ids.shape, hidden] -> fp32 gradient of the table, written to `out` whole or, with accumulate, added to it"""
        cfg = self._cfg(ids, gx.GX_ACCUM_WGRAD if accumulate else 0)
        self._check("dy", dy, (*ids.shape, self.hidden), self.tdtype)
        _need(out is not None or not accumulate, "accumulate: into which gradient?")
        if out is None:
            out = self._new((self.rows, self.hidden), torch.float32)
        else:
            self._check("out", out, (self.rows, self.hidden), torch.float32)
        stream = self._stream()
        gx.embed_bwd(cfg, ids, dy, out, self._workspace(gx.embed_workspace_bytes(cfg), stream), stream)
        return out


class DeviceHeadNorm(_Operator):
    """RMS norm of every query and key head with a gain per column, then the rotation of the first `rot_dim` columns by the
    token's position; columns (i, i + rot_dim / 2) turn together, or with `pairs` (2 i, 2 i + 1).  A token whose position the
    tables of angles do not have becomes NaN."""

    def __init__(self, head_dim, rot_dim=0, dtype="bf16", eps=1e-6, pairs=False, device="cuda:0"):
        super().__init__(dtype, device)
        self.head_dim, self.rot_dim, self.eps, self.pairs = head_dim, rot_dim, eps, pairs

    def _side(self, name, x, gain, pos):
        shape = self._heads(name, x)
        if gain is not None:
            self._check(name + " gain", gain, (self.head_dim,), self.tdtype)
        if pos is not None:
            self._check(name + " positions", pos, shape[:2], torch.int32)
        return shape

    def _args(self, q, k, gain_q, gain_k, cos, sin, q_pos, k_pos, flags):
        _need(q is not None or k is not None, "queries or keys")
        b = sq = hq = sk = hk = max_pos = 0
        if q is not None:
            b, sq, hq, _ = self._side("q", q, gain_q, q_pos)
        if k is not None:
            bk, sk, hk, _ = self._side("k", k, gain_k, k_pos)
            _need(q is None or b == bk, "queries and keys of as many samples")
            b = bk
        if self.rot_dim:
            _need(cos is not None and sin is not None, "tables of cosines and sines")
            max_pos = cos.shape[0]
            shape = (max_pos, self.rot_dim // 2)
            self._check("cos", cos, shape, torch.float32)
            self._check("sin", sin, shape, torch.float32)
        else:
            cos = sin = None
        cfg = gx.HeadsNormCfg(b, sq, sk, hq, hk, self.head_dim, self.rot_dim, max_pos, self.gtype,
                              flags | gx.GX_ROPE_PAIRS if self.pairs else flags, self.eps)
        return cfg, gx.heads_norm_in(q, k, gain_q, gain_k, q_pos, k_pos, cos, sin)

    def _like(self, name, x, given):
        """Where the result for x goes: `given`, or a new tensor"""
        if x is None:
            return None
        if given is None:
            return torch.empty_like(x)
        self._check(name, given, x.shape, self.tdtype, False)
        return given

    def _gain_like(self, name, x, gain, given, accumulate):
        if x is None or gain is None:
            return None
        if given is None:
            _need(not accumulate, f"accumulate: into which {name}?")
            return torch.empty_like(gain, dtype=torch.float32)
        self._check(name, given, (self.head_dim,), torch.float32)
        return given

    def forward(self, q, k=None, gain_q=None, gain_k=None, cos=None, sin=None, q_pos=None, k_pos=None, q_out=None, k_out=None):
        """q [batch, tokens, heads, head_dim], k the same with its own tokens and heads, or either None; positions int32 [batch,
        tokens] (None: 0, 1, ...); cos, sin fp32 [positions, rot_dim / 2].  Returns (q, k), normed and turned; q_out, k_out
        may be q and k themselves."""
        cfg, inputs = self._args(q, k, gain_q, gain_k, cos, sin, q_pos, k_pos, 0)
        q_out, k_out = self._like("q_out", q, q_out), self._like("k_out", k, k_out)
        gx.heads_norm_fwd(cfg, inputs, q_out, k_out, self._stream())
        return q_out, k_out

    def backward(self, q, k, dq_out, dk_out, gain_q=None, gain_k=None, cos=None, sin=None, q_pos=None, k_pos=None, dq=None, dk=None,
                 dgain_q=None, dgain_k=None, accumulate=False):
        """The forward pass's inputs and the gradients of its outputs -> (dq, dk, dgain_q, dgain_k); the gains' are fp32, None
        without a gain, and added to with accumulate."""
        cfg, inputs = self._args(q, k, gain_q, gain_k, cos, sin, q_pos, k_pos, gx.GX_ACCUM_WGRAD if accumulate else 0)
        if q is not None:
            self._check("dq_out", dq_out, q.shape, self.tdtype, False)
        if k is not None:
            self._check("dk_out", dk_out, k.shape, self.tdtype, False)
        dq, dk = self._like("dq", q, dq), self._like("dk", k, dk)
        dgain_q = self._gain_like("dgain_q", q, gain_q, dgain_q, accumulate)
        dgain_k = self._gain_like("dgain_k", k, gain_k, dgain_k, accumulate)
        stream = self._stream()
        ws = self._workspace(gx.heads_norm_workspace_bytes(cfg), stream)
        gx.heads_norm_bwd(cfg, inputs, dq_out if q is not None else None, dk_out if k is not None else None, dq, dk, dgain_q, dgain_k,
                          ws, stream)
        return dq, dk, dgain_q, dgain_k


class DeviceCrossAttention(_Operator):
    """softmax(scale Q K^T over the keys that count) V for queries and keys of different sequences; query head h reads key head
    h // (query heads / key heads).  scale: 1 / sqrt(head_dim) unless given."""

    def __init__(self, head_dim, dtype="bf16", scale=None, device="cuda:0"):
        super().__init__(dtype, device)
        self.head_dim, self.scale = head_dim, head_dim ** -0.5 if scale is None else scale

    def _args(self, q, k, v, key_lens, key_mask):
        b, n, hq, _ = self._heads("q", q)
        bk, m, hk, _ = shape = self._heads("k", k)
        _need(bk == b and self._heads("v", v) == shape, "keys and values of one shape, as many samples as queries")
        if key_lens is not None:
            self._check("key_lens", key_lens, (b,), torch.int32)
        if key_mask is not None:
            _need(key_mask.dtype in (torch.bool, torch.uint8), f"key_mask: {key_mask.dtype}, not bool or uint8")
            self._check("key_mask", key_mask, (b, m), key_mask.dtype)
        cfg = gx.CrossCfg(b, n, m, hq, hk, self.head_dim, self.gtype, 0, self.scale)
        return cfg, gx.cross_in(q, k, v, key_lens, key_mask)

    def forward(self, q, k, v, key_lens=None, key_mask=None, want_lse=True, out=None):
        """q [batch, queries, heads, head_dim], k, v [batch, keys, key heads, head_dim], key_lens int32 [batch], key_mask bool or bytes
        [batch, keys] -> (o, lse); lse fp32 [batch, heads, queries] is for the backward pass, None without want_lse"""
        cfg, inputs = self._args(q, k, v, key_lens, key_mask)
        if out is None:
            out = torch.empty_like(q)
        else:
            self._check("out", out, q.shape, self.tdtype, False)
        lse = self._new((q.shape[0], q.shape[2], q.shape[1]), torch.float32) if want_lse else None
        stream = self._stream()
        nbytes = gx.cross_workspace_bytes(cfg, False)
        gx.cross_fwd(cfg, inputs, out, lse, self._workspace(nbytes, stream) if nbytes else None, stream)
        return out, lse

    def backward(self, q, k, v, o, lse, do, key_lens=None, key_mask=None, dq=None, dk=None, dv=None):
        """The forward pass's inputs and outputs and the gradient of o -> (dq, dk, dv)"""
        cfg, inputs = self._args(q, k, v, key_lens, key_mask)
        b, n, hq, _ = shape = q.shape
        self._check("o", o, shape, self.tdtype, False)
        self._check("do", do, shape, self.tdtype, False)
        self._check("lse", lse, (b, hq, n), torch.float32)
        if dq is None:
            dq = torch.empty_like(q)
        else:
            self._check("dq", dq, shape, self.tdtype, False)
        if dk is None:
            dk = torch.empty_like(k)
        else:
            self._check("dk", dk, k.shape, self.tdtype, False)
        if dv is None:
            dv = torch.empty_like(v)
        else:
            self._check("dv", dv, k.shape, self.tdtype, False)
        stream = self._stream()
        ws = self._workspace(gx.cross_workspace_bytes(cfg, True), stream)
        gx.cross_bwd(cfg, inputs, o, lse, do, dq, dk, dv, ws, stream)
        return dq, dk, dv
