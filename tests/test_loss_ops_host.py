"""What the losses of logits refuse, and with which status, before anything reaches a GPU; sizes of their scratch."""
import os

import pytest
import torch

from paper_2504_03662_amd import binding as gx

P = 1 << 20                                # an address that is never followed: every call here ends before a launch


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(gx.LIB_PATH):
        from paper_2504_03662_amd.build import build
        build(verbose=False)
    return gx.lib()


def _cfg(**kw):
    d = dict(rows=10, vocab=100, dtype=gx.GX_BF16, id_bytes=8, flags=0, scale=1.0, stride=100, grad_stride=100, first_id=0, whole_vocab=0,
             ignore_id=-1)
    d.update(kw)
    return gx.LogitsCfg(*d.values())


def _policy(low=0.2, high=0.2, kl=0.1, flags=0):
    return gx.PolicyCfg(low, high, kl, flags)


def _pairs(pairs=2, rows=10, beta=0.1, margin=0.0, smoothing=0.0, flags=0):
    return gx.PairsCfg(pairs, rows, beta, margin, smoothing, flags)


def _distill(top=4, dtype=gx.GX_F32, flags=0):
    return gx.DistillCfg(top, dtype, flags)


IN = gx.policy_in(P, P, P, P)
CALLS = dict(
    logp_fwd=lambda c, z=P, ids=P, a=P, b=P: gx.logp_fwd(c, z, ids, a, b, check=False),
    logp_bwd=lambda c, z=P, ids=P, a=P, b=P, d=P: gx.logp_bwd(c, z, ids, a, b, d, check=False),
    token=lambda c, z=P, ids=P, a=P, b=P, d=P: gx.token_loss(c, z, ids, P, a, b, d, check=False),
    policy=lambda c, z=P, ids=P, a=P, b=P, d=P: gx.policy_loss(c, _policy(), IN, z, ids, a, b, d, check=False),
    preference=lambda c, z=P, ids=P, a=P, b=P, d=P: gx.preference_loss(c, _pairs(), IN, z, ids, a, b, d, P, check=False),
    distill=lambda c, z=P, ids=P, a=P, d=P: gx.distill_loss(c, _distill(), gx.distill_in(ids, P, P, P), z, a, d, P, check=False))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 2), (dict(rows=(1 << 21) + 1), 2), (dict(vocab=0), 2), (dict(vocab=(1 << 19) + 1, stride=1 << 20, grad_stride=1 << 20), 2),
    (dict(stride=99), 2), (dict(grad_stride=99), 2), (dict(stride=1 << 41), 2), (dict(scale=0.0), 2), (dict(scale=-1.0), 2),
    (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2), (dict(scale=1e-9), 2), (dict(first_id=-1), 2), (dict(first_id=5), 2),
    (dict(whole_vocab=99), 2), (dict(first_id=100, whole_vocab=199), 2), (dict(dtype=2), 4), (dict(id_bytes=2), 4), (dict(flags=16), 6)])
def test_configurations(name, kw, status):
    assert CALLS[name](_cfg(**kw)) == status
    assert gx.preference_workspace_bytes(_cfg(**kw)) == 0


@pytest.mark.parametrize("name", CALLS)
def test_pointers(name):
    call, c = CALLS[name], _cfg()
    for k, kw in enumerate((dict(z=None), dict(ids=None), dict(a=None))):
        assert call(c, **kw) == 1
    for kw in (dict(z=P + 1), dict(ids=P + 4), dict(a=P + 2)):
        assert call(c, **kw) == 5
    assert call(_cfg(dtype=gx.GX_F32), z=P + 2) == 5
    if name != "distill":
        assert call(c, b=P + 2) == 5
    if name != "logp_fwd":
        assert call(c, d=P + 1) == 5
        assert call(_cfg(dtype=gx.GX_F32), d=P + 2) == 5
    if not torch.cuda.is_available():                              # the last check before a launch
        reached = 7
        assert call(c) == call(_cfg(id_bytes=4), ids=P + 4) == call(c, z=P + 2) == reached
        if name in ("token", "policy", "preference"):
            assert call(c, b=None, d=None) == reached
        if name == "logp_fwd":
            assert call(c, b=None) == reached
    if name == "logp_bwd":
        assert call(c, b=None) == call(c, d=None) == 1


def test_shards_are_for_log_probabilities():
    c = _cfg(first_id=100, whole_vocab=300)
    for name, call in CALLS.items():
        if not name.startswith("logp"):
            assert call(c) == 2
        elif not torch.cuda.is_available():
            assert call(c) == 7


@pytest.mark.parametrize("kw,status", [(dict(low=-0.1), 2), (dict(low=1.5), 2), (dict(low=float("nan")), 2), (dict(high=-0.1), 2),
                                       (dict(high=float("inf")), 2), (dict(kl=-1.0), 2), (dict(kl=float("nan")), 2), (dict(flags=1), 6)])
def test_policy(kw, status):
    assert gx.policy_loss(_cfg(), _policy(**kw), IN, P, P, P, P, P, check=False) == status


def test_policy_inputs():
    call = lambda i, kl=0.1: gx.policy_loss(_cfg(), _policy(kl=kl), i, P, P, P, P, P, check=False)
    assert call(gx.policy_in(None, P, P)) == call(gx.policy_in(P, None, P)) == call(gx.policy_in(P, P, None)) == 1
    assert call(gx.policy_in(P + 2, P, P)) == call(gx.policy_in(P, P + 2, P)) == call(gx.policy_in(P, P, P, P + 1)) == 5
    assert gx.policy_loss(_cfg(), None, IN, P, P, P, P, P, check=False) == 1
    if not torch.cuda.is_available():
        assert call(gx.policy_in(P, P, None, None), kl=0.0) == 7
    with pytest.raises(gx.GxError, match="gx_policy_loss"):
        gx.policy_loss(_cfg(), _policy(), None, P, P, P, P, P)


@pytest.mark.parametrize("kw,status", [(dict(pairs=-1), 2), (dict(pairs=(1 << 20) + 1), 2), (dict(rows=-1), 2), (dict(smoothing=-0.1), 2),
                                       (dict(smoothing=1.1), 2), (dict(smoothing=float("nan")), 2), (dict(beta=float("inf")), 2),
                                       (dict(margin=float("nan")), 2), (dict(flags=4), 6)])
def test_pairs(kw, status):
    assert gx.pairs_loss(_pairs(**kw), IN, P, P, P, P, check=False) == status
    assert gx.preference_loss(_cfg(), _pairs(**kw), IN, P, P, P, P, P, P, check=False) == status


def test_pairs_inputs():
    c = _pairs()
    assert gx.pairs_loss(c, None, P, P, P, P, check=False) == 1
    assert gx.pairs_loss(c, gx.pairs_in(None), P, P, P, P, check=False) == 1
    assert gx.pairs_loss(c, IN, None, P, P, P, check=False) == gx.pairs_loss(c, IN, P, None, P, P, check=False) == 1
    assert gx.pairs_loss(c, gx.pairs_in(P + 2), P, P, P, P, check=False) == 5
    assert gx.pairs_loss(c, IN, P, P, P, P + 2, check=False) == 5
    assert gx.pairs_loss(_pairs(pairs=0, rows=0), gx.pairs_in(P), None, None, None, None, check=False) == gx.GX_OK
    assert gx.preference_loss(_cfg(), _pairs(rows=9), IN, P, P, P, P, P, P, check=False) == 2      # not the logits' rows
    assert gx.preference_loss(_cfg(), c, IN, P, P, P, P, P, None, check=False) == 1
    assert gx.preference_loss(_cfg(), c, IN, P, P, P, P, P, P + 8, check=False) == 5
    if not torch.cuda.is_available():
        assert gx.pairs_loss(c, gx.pairs_in(P), P, P, None, None, check=False) == 7


def test_distillation():
    call = lambda c, i, ws=P: gx.distill_loss(_cfg(), c, i, P, P, P, ws, check=False)
    for kw, status in ((dict(top=0), 2), (dict(top=1025), 2), (dict(dtype=3), 4), (dict(flags=1), 6)):
        assert call(_distill(**kw), IN) == status
        assert gx.distill_workspace_bytes(_cfg(), _distill(**kw)) == gx.distill_workspace_bytes(_cfg(rows=-1), _distill()) == 0
    assert call(_distill(), IN, None) == 1 and call(_distill(), IN, P + 8) == 5
    # a record of every entry
    assert gx.distill_workspace_bytes(_cfg(rows=1000), _distill(top=64)) >= 1000 * 64 * 16
    assert call(_distill(), gx.distill_in(None, P)) == call(_distill(), gx.distill_in(P, None)) == call(None, IN) == 1
    assert call(_distill(), gx.distill_in(P, P + 2)) == call(_distill(), gx.distill_in(P, P, P + 2)) == 5
    if not torch.cuda.is_available():
        assert call(_distill(dtype=gx.GX_BF16), gx.distill_in(P, P + 2)) == 7


def test_nothing_to_do():
    none = _cfg(rows=0)
    assert gx.logp_fwd(none, None, None, None, None, check=False) == gx.GX_OK
    assert gx.logp_bwd(none, None, None, None, None, None, check=False) == gx.GX_OK
    assert gx.token_loss(none, None, None, None, None, None, None, check=False) == gx.GX_OK
    assert gx.policy_loss(none, _policy(), IN, None, None, None, None, None, check=False) == gx.GX_OK
    assert gx.distill_loss(none, _distill(), IN, None, None, None, None, check=False) == gx.GX_OK


def test_scratch_grows_with_rows():
    sizes = [gx.preference_workspace_bytes(_cfg(rows=n)) for n in (1, 17, 1000, 1 << 21)]
    assert sizes == sorted(sizes) and sizes[2] >= 1000 * 24


# ---- the classes on torch tensors: nothing below reaches the library's launch -------------------------------------------------

from paper_2504_03662_amd import loss_ops as ops  # noqa: E402


def _tensors(rows=4, vocab=10):
    return torch.zeros(rows, vocab), torch.zeros(rows, dtype=torch.long), torch.zeros(rows)


def test_classes_check_shapes_types_and_devices():
    z, ids, f = _tensors()
    op = ops.DeviceTokenLoss(10, "f32", device="cpu")
    for bad, match in (((torch.zeros(4, 11), ids), "logits"), ((z.bfloat16(), ids), "logits: torch.bfloat16"), ((z, ids[:3]), "ids: shape"),
                       ((z, ids.short()), "ids: torch.int16"), ((z, ids, f.double()), "weights: torch.float64"),
                       ((z, ids, f[:2]), "weights: shape"), ((torch.zeros(4, 20)[:, ::2], ids), "columns are not contiguous"),
                       ((torch.zeros(10), ids[:1]), "logits"), ((torch.zeros(3, 4, 10)[:, :2], torch.zeros(3, 2, dtype=torch.long)), "distance"),
                       ((torch.zeros(1, 10).expand(4, 10), ids), "overlap")):
        with pytest.raises(ValueError, match=match):
            op.forward(*bad)
    with pytest.raises(ValueError, match="out: shape"):
        op.forward_backward(z, ids, out=torch.zeros(4, 11))
    with pytest.raises(ValueError, match="lse: shape"):
        op.logp_backward(z, ids, f[:1], f)
    with pytest.raises(ValueError, match="dlogp: torch.float64"):
        op.logp_backward(z, ids, f, f.double())
    policy = ops.DevicePolicyLoss(10, "f32", kl=0.1, device="cpu")
    with pytest.raises(ValueError, match="ref_logp"):
        policy.forward(z, ids, f, f)
    with pytest.raises(ValueError, match="advantages: shape"):
        policy.forward(z, ids, f, f[:1], f)
    pref = ops.DevicePreferenceLoss(10, "f32", device="cpu")
    for starts, match in ((torch.zeros(4, dtype=torch.int32), "starts"), (torch.zeros(3, dtype=torch.long), "starts: torch.int64"),
                          (torch.zeros(1, 3, dtype=torch.int32), "starts")):
        with pytest.raises(ValueError, match=match):
            pref.forward(z, ids, starts)
    with pytest.raises(ValueError, match="pair_weights: shape"):
        pref.forward(z, ids, torch.zeros(3, dtype=torch.int32), pair_weights=f)
    distill = ops.DeviceDistillation(10, "f32", device="cpu")
    top = torch.zeros(4, 3, dtype=torch.long)
    for bad, match in (((z, top[:3], torch.zeros(3, 3)), "top_ids"), ((z, top, torch.zeros(4, 2)), "top_logits: shape"),
                       ((z, top, torch.zeros(4, 3).half()), "top_logits: torch.float16"), ((z, top, torch.zeros(4, 3), f[:1]), "top_lse"),
                       ((z, top.t().contiguous().t(), torch.zeros(4, 3)), "ids: not contiguous")):
        with pytest.raises(ValueError, match=match):
            distill.forward(*bad)


def test_rows_of_views():
    op = ops.DeviceTokenLoss(10, "f32", device="cpu")
    assert op._rows("z", torch.zeros(4, 10)) == 10 and op._rows("z", torch.zeros(4, 16)[:, 3:13]) == 16
    assert op._rows("z", torch.zeros(2, 3, 16)[..., :10]) == 16 and op._rows("z", torch.zeros(1, 3, 7, 10)[:, :, 2]) == 70
    assert op._rows("z", torch.zeros(5, 16)[2:3, :10]) == 10
    whole = torch.zeros(6, 5, 17)[..., 1:11]
    out, stride = op._gradient(whole, 17, None)
    assert out.shape == whole.shape and out.stride() == (5 * stride, stride, 1) and (stride - 17) % 4 == 0 and stride >= 10
    assert out.storage_offset() == whole.data_ptr() % 16 // 4
    out.fill_(1.0)                                                  # within its memory


@pytest.mark.parametrize("make", [ops.DeviceTokenLoss, ops.DevicePolicyLoss, ops.DevicePreferenceLoss, ops.DeviceDistillation])
def test_work_goes_to_the_operators_gpu_or_nowhere(make, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="cuda:1"):
        make(10, device="cuda:1")._stream()


@pytest.mark.parametrize("dtype,rows", [(gx.GX_F32, 1 << 17), (gx.GX_BF16, 1 << 18)])
def test_too_many_pieces_are_refused_before_any_launch(dtype, rows):
    """2^24 pieces of rows of 2^19 columns, in the two gradients that are cut into pieces"""
    cfg = _cfg(rows=rows, vocab=1 << 19, stride=1 << 19, grad_stride=1 << 19, dtype=dtype)
    assert gx.logp_bwd(cfg, P, P, P, P, P, check=False) == 2
    assert gx.preference_loss(cfg, _pairs(rows=rows), gx.pairs_in(P, P, P, P), P, P, P, P, P, P, check=False) == 2
