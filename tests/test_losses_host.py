"""The loss operators without a GPU: what the library refuses on the host, before any launch, and
what the binding refuses; the 64-bit references against finite differences."""
import ctypes
import math

import numpy as np
import pytest

import _losses as ref
import paper_2606_19989_amd as odb

P = 0x100000    # a pointer that is never dereferenced: every call below ends in its host checks
byref = ctypes.byref


def _logits(**kw):
    return odb.Logits(**{**dict(dtype=1, shift=1, rows=2, cols=3, vocab=10, row_stride=30, col_stride=10, scale=1.0,
                                d_logits=P), **kw})


BAD_LOGITS = [dict(dtype=3), dict(dtype=-1), dict(shift=2), dict(shift=-1), dict(rows=-1), dict(cols=-1),
              dict(rows=1 << 16, cols=1 << 15), dict(rows=1 << 62, cols=4), dict(vocab=0), dict(vocab=1 << 31),
              dict(row_stride=-1), dict(col_stride=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
              dict(scale=math.inf), dict(scale=1e-60), dict(scale=3e38), dict(d_logits=None), dict(d_logits=P + 1),
              dict(dtype=0, d_logits=P + 2), dict(row_stride=1 << 62), dict(col_stride=1 << 61)]


@pytest.mark.parametrize("bad", BAD_LOGITS, ids=str)
def test_logits_refused(bad):
    lib = odb.load()
    x = _logits(**bad)
    assert lib.odb_token_logprobs(byref(x), P, P, P, None, None, None) == odb.ODB_E_INVALID_ARG
    assert lib.odb_last_error_message() != b""
    assert lib.odb_token_logprobs_backward(byref(x), P, P, P, None, None, P + 4096, 30, 10, None, None) == \
        odb.ODB_E_INVALID_ARG


def test_logprobs_arguments_refused():
    lib = odb.load()
    x = _logits()
    assert lib.odb_token_logprobs(None, P, P, P, None, None, None) == odb.ODB_E_INVALID_ARG
    assert lib.odb_token_logprobs(byref(x), None, P, P, None, None, None) == odb.ODB_E_INVALID_ARG
    assert lib.odb_token_logprobs(byref(x), P, None, P, None, None, None) == odb.ODB_E_INVALID_ARG
    assert lib.odb_token_logprobs(byref(x), P, P, P + 4, None, None, None) == odb.ODB_E_INVALID_ARG
    bwd = lambda labels=P, stats=P, g=P, ent=None, ge=None, out=P + 4096, rs=30, cs=10, x=x: \
        lib.odb_token_logprobs_backward(byref(x), labels, stats, g, ent, ge, out, rs, cs, None, None)
    for bad in (dict(labels=None), dict(stats=None), dict(stats=P + 4), dict(g=None), dict(ent=P), dict(ge=P),
                dict(out=None), dict(out=P + 1), dict(rs=-1), dict(cs=-1),
                dict(cs=9), dict(rs=29), dict(rs=10, cs=10), dict(rs=0), dict(rs=10, cs=19),   # elements overlap
                dict(out=P, rs=40), dict(out=P, rs=40, cs=12)):                                # in place, other strides
        assert bwd(**bad) == odb.ODB_E_INVALID_ARG, bad
    # nothing to do: no launch, no pointers needed
    for shape in (dict(rows=0), dict(cols=0)):
        x0 = _logits(d_logits=None, **shape)
        assert lib.odb_token_logprobs(byref(x0), None, None, None, None, None, None) == odb.ODB_OK
        assert lib.odb_token_logprobs_backward(byref(x0), None, None, None, None, None, None, 30, 10, None, None) == \
            odb.ODB_OK


def _tiles(**kw):
    return odb.TilesStruct(**{**dict(num_slots=2, num_rows=5, num_elems=50, d_slot_rows=P, d_slot_maxlen=P,
                                     d_slot_row_off=P, d_slot_tile_off=P, d_labels=P, shift=1), **kw})


BAD_TILES = [dict(num_slots=-1), dict(num_slots=1 << 31), dict(num_rows=-1), dict(num_rows=1 << 31),
             dict(num_elems=-1), dict(num_elems=(1 << 36) + 1), dict(num_elems=(1 << 63) - 1), dict(shift=2),
             dict(shift=-1), dict(reserved0=1)]
BAD_ARRAYS = [dict(d_slot_rows=None), dict(d_slot_maxlen=None), dict(d_slot_row_off=None), dict(d_slot_tile_off=None),
              dict(d_labels=None)]


def _policy(t=None, p=None, ws=P, ws_bytes=1 << 40, **kw):
    a = {**dict(lp=P, old=P, ref=P, ent=None, adv=P, w=None, loss=P, means=P, counts=P, g=P, ge=None), **kw}
    return odb.load().odb_policy_loss(byref(t or _tiles()), byref(p or odb.PolicyParams(kl=3)), *a.values(), None, ws,
                                      ws_bytes, None)


def _preference(t=None, p=None, ws=P, ws_bytes=1 << 40, **kw):
    a = {**dict(lp=P, ref=P, ids=P, num=9, pair=P, loss=P, row_loss=P, reward=P, counts=P, g=P), **kw}
    return odb.load().odb_preference_loss(byref(t or _tiles()), byref(p or odb.PreferenceParams()), *a.values(), None,
                                          ws, ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_TILES + BAD_ARRAYS, ids=str)
def test_tiles_refused(bad):
    t = _tiles(**bad)
    if bad not in BAD_ARRAYS:
        assert odb.load().odb_loss_workspace_size(byref(t), 0) == 0
    assert _policy(t) == odb.ODB_E_INVALID_ARG
    assert _preference(t) == odb.ODB_E_INVALID_ARG


def test_loss_workspace():
    lib = odb.load()
    size = lambda ids=0, **kw: lib.odb_loss_workspace_size(byref(_tiles(**kw)), ids)
    assert lib.odb_loss_workspace_size(None, 0) == 0
    assert size(-1) == 0 and size(1 << 31) == 0
    assert 0 < size() <= size(100) and size(10 ** 6) >= size() + 4 * 10 ** 6 - 4096
    assert size(num_elems=1 << 36) > (1 << 33)
    need = size()
    for call, n in ((_policy, need), (_preference, size(9))):
        assert call(ws=None) == odb.ODB_E_INVALID_ARG
        assert call(ws=P + 8) == odb.ODB_E_INVALID_ARG
        assert call(ws_bytes=n - 1) == odb.ODB_E_WORKSPACE


def test_policy_arguments_refused():
    lib = odb.load()
    for bad in (dict(kl=-1), dict(kl=4), dict(reduce=3), dict(reduce=-1), dict(token_advantage=2), dict(reserved0=1),
                dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=math.nan), dict(clip_high=-0.1),
                dict(clip_high=math.nan), dict(dual_clip=1.0), dict(dual_clip=-1.0), dict(dual_clip=math.inf),
                dict(dual_clip=math.nan), dict(kl_coef=math.nan), dict(entropy_coef=math.inf),
                dict(loss_scale=math.nan), dict(entropy_coef=0.1)):     # an entropy term without entropies
        assert _policy(p=odb.PolicyParams(**bad)) == odb.ODB_E_INVALID_ARG, bad
    for bad in ("lp", "ref", "adv", "loss", "means", "counts"):
        assert _policy(**{bad: None}) == odb.ODB_E_INVALID_ARG, bad
    assert _policy(ge=P) == odb.ODB_E_INVALID_ARG
    t = _tiles(num_slots=0, d_slot_rows=None)
    assert _policy(t, ws=None) == odb.ODB_OK       # nothing to do
    assert lib.odb_policy_loss(byref(_tiles()), None, *[P] * 11, None, P, 1 << 40, None) == odb.ODB_E_INVALID_ARG


def test_policy_coefficients_beyond_fp32_refused():
    for big in (1e39, -1e39, 3.4028236e38):     # the last one rounds to infinity
        assert _policy(p=odb.PolicyParams(kl=3, kl_coef=big)) == odb.ODB_E_INVALID_ARG, big
        assert _policy(p=odb.PolicyParams(kl=3, entropy_coef=big), ent=P) == odb.ODB_E_INVALID_ARG, big


def test_preference_arguments_refused():
    for bad in (dict(kind=3), dict(kind=-1), dict(normalize=2), dict(beta=0.0), dict(beta=-1.0), dict(beta=math.nan),
                dict(beta=math.inf), dict(margin=math.nan), dict(loss_scale=math.inf), dict(label_smoothing=-0.1),
                dict(label_smoothing=1.5), dict(label_smoothing=math.nan), dict(kind=1, label_smoothing=0.1),
                dict(kind=2, label_smoothing=0.1)):
        assert _preference(p=odb.PreferenceParams(**bad)) == odb.ODB_E_INVALID_ARG, bad
    for bad in ("lp", "pair", "loss", "row_loss", "reward", "counts"):
        assert _preference(**{bad: None}) == odb.ODB_E_INVALID_ARG, bad
    assert _preference(num=-1) == odb.ODB_E_INVALID_ARG
    assert _preference(num=1 << 31) == odb.ODB_E_INVALID_ARG
    assert _preference(ids=None, num=6) == odb.ODB_E_INVALID_ARG      # rows are their own ids


def test_binding_refuses_host_tensors():
    import torch

    z = torch.zeros(1, 2, 5)
    y = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        odb.odb_token_logprobs(z, y, torch.zeros(1, 2))
    with pytest.raises(ValueError):
        odb.odb_token_logprobs(z.double(), y, torch.zeros(1, 2))
    with pytest.raises(ValueError):
        odb.odb_token_logprobs(z[0], y, torch.zeros(1, 2))
    with pytest.raises(ValueError):
        odb.odb_token_logprobs(z.transpose(1, 2), y, torch.zeros(1, 2))
    i32, i64 = dict(dtype=torch.int32), dict(dtype=torch.int64)
    with pytest.raises(ValueError):
        odb.Tiles(torch.zeros(1, **i32), torch.zeros(1, **i32), torch.zeros(2, **i64), torch.zeros(2, **i64), y, 1)


def test_binding_refuses_arrays_of_a_transposed_tile():
    import types

    import torch

    tile, f32 = types.SimpleNamespace(rows=4, cols=9), torch.float32
    array = lambda *shape, each=1: odb._tile_array(torch.zeros(*shape), f32, tile, "stats", -1, each)   # -1: the host
    for shape in ((9, 4), (2, 18), (9, 4, 1), (5, 9)):
        with pytest.raises(ValueError, match="stats"):
            array(*shape)
    with pytest.raises(ValueError, match="stats"):
        array(9, 4, 2, each=2)
    for shape in ((4, 9), (36,), (40,), (1, 36), (36, 1), (4, 9, 1), (4, 3, 3), (1, 4, 9)):
        assert array(*shape)
    for shape in ((4, 9, 2), (36, 2), (72,), (1, 72)):
        assert array(*shape, each=2)


def test_tiles_of_a_plan_refuse_labels_with_strides():
    import torch

    plan = odb._PlanLosses()
    plan.torch, plan.outputs, plan.num_slots = torch, None, 2
    plan.info = {"emitted_samples": 3, "padded_elems": 20}
    # a copy of them would be made on the current stream and not on the loss's
    with pytest.raises(ValueError, match="contiguous"):
        plan.tiles(torch.zeros(5, 8, dtype=torch.int32)[:, ::2])


# ------------------------------------------------------------ the references themselves
def _difference(f, x, at, eps):
    up, down = x.copy(), x.copy()
    up[at] += eps
    down[at] -= eps
    return (f(up) - f(down)) / (2 * eps)


def test_reference_logprob_gradient_is_the_difference():
    rng = np.random.default_rng(3)
    z = rng.normal(size=(2, 3, 7)) * 2
    y = np.array([[1, 6, ref.IGNORE], [0, 2, 5]])
    g, h = rng.normal(size=(2, 3)), rng.normal(size=(2, 3))

    def value(z):
        lp, _, ent, _, _ = ref.token_logprobs(z, y, 1, 0.7)
        return (g * lp + h * ent).sum()
    got = ref.token_logprobs_grad(z, y, 1, 0.7, g, h)
    for at in np.ndindex(z.shape):
        assert abs(got[at] - _difference(value, z, at, 1e-5)) < 1e-8, at


@pytest.mark.parametrize("kl", range(4))
@pytest.mark.parametrize("reduce", range(3))
def test_reference_policy_gradient_is_the_difference(kl, reduce):
    rng = np.random.default_rng(5)
    plan = ref.Plan([[4, 6], [], [9]])
    y = plan.labels(rng, 0.3)
    lp, H = -rng.random(plan.E) * 3, rng.random(plan.E)
    old, kref, adv = lp + rng.normal(size=plan.E) * 0.3, lp + rng.normal(size=plan.E), rng.normal(size=plan.R)
    p = dict(kl=kl, reduce=reduce, token_advantage=0, clip_low=0.2, clip_high=0.3, dual_clip=1.5, kl_coef=0.1,
             entropy_coef=0.05, loss_scale=2.0)
    w = np.array([0.3, 0.2, 0.5])
    value = lambda lp, H: ref.policy_loss(plan, y, 1, p, lp, old, kref, H, adv, w)["loss"].sum()
    r = ref.policy_loss(plan, y, 1, p, lp, old, kref, H, adv, w)
    for e in range(plan.E):
        # the steps stay on one side of every clip
        assert abs(r["grad"][e] - _difference(lambda v: value(v, H), lp, e, 1e-6)) < 1e-7, e
        assert abs(r["grad_ent"][e] - _difference(lambda v: value(lp, v), H, e, 1e-6)) < 1e-8, e


@pytest.mark.parametrize("kind", range(3))
@pytest.mark.parametrize("normalize", [0, 1])
def test_reference_preference_gradient_is_the_difference(kind, normalize):
    rng = np.random.default_rng(6)
    plan = ref.Plan([[3, 5], [2], [4, 4, 6]])
    y = plan.labels(rng, 0.3)
    lp, kref = -rng.random(plan.E) * 2, -rng.random(plan.E) * 2
    p = dict(kind=kind, normalize=normalize, beta=0.4, margin=0.1, label_smoothing=0.1 if kind == 0 else 0.0,
             loss_scale=0.5)
    ids, pair = np.array([4, 1, 0, 2, 5, 3]), np.array([5 + 1, -(2 + 1), 1 + 1, 0, 0, -(0 + 1)])
    value = lambda lp: ref.preference_loss(plan, y, 1, p, lp, kref, ids, pair)["loss"]
    r = ref.preference_loss(plan, y, 1, p, lp, kref, ids, pair)
    assert r["counts"][0] == 2
    for e in range(plan.E):
        assert abs(r["grad"][e] - _difference(value, lp, e, 1e-6)) < 1e-7, e
