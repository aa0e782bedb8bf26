"""The operators over lists of tokens without a GPU: what the library and the binding refuse before any launch."""
import ctypes

import numpy as np
import pytest

import _lists as ref
import paper_2606_19989_amd as odb
from test_losses_host import BAD_LOGITS, P, _logits

byref = ctypes.byref
BAD = odb.ODB_E_INVALID_ARG


def _list(x=None, labels=P, k=4, ids=P, out=P, stats=P):
    return odb.load().odb_token_list_logprobs(byref(_logits() if x is None else x), labels, k, ids, out, stats, None, None)


def _list_back(x=None, labels=P, k=4, ids=P, stats=P, g=P, out=P + 4096, rs=30, cs=10):
    return odb.load().odb_token_list_logprobs_backward(byref(_logits() if x is None else x), labels, k, ids, stats, g,
                                                       out, rs, cs, None, None)


@pytest.mark.parametrize("bad", BAD_LOGITS, ids=str)
def test_logits_refused(bad):
    assert _list(_logits(**bad)) == BAD and odb.load().odb_last_error_message() != b""
    assert _list_back(_logits(**bad)) == BAD


def test_list_arguments_refused():
    assert odb.load().odb_token_list_logprobs(None, P, 4, P, P, P, None, None) == BAD
    assert odb.load().odb_token_list_logprobs_backward(None, P, 4, P, P, P, P, 30, 10, None, None) == BAD
    for bad in (dict(k=0), dict(k=-1), dict(k=odb.ODB_LIST_MAX + 1), dict(ids=None), dict(out=None), dict(stats=P + 4)):
        assert _list(**bad) == BAD, bad
    for bad in (dict(k=0), dict(k=odb.ODB_LIST_MAX + 1), dict(ids=None), dict(stats=None), dict(stats=P + 4),
                dict(g=None), dict(out=None), dict(out=P + 1), dict(rs=-1), dict(cs=-1), dict(cs=9), dict(rs=29),
                dict(rs=10, cs=10), dict(rs=0), dict(out=P, rs=40), dict(out=P, rs=40, cs=12)):
        assert _list_back(**bad) == BAD, bad
    for shape in (dict(rows=0), dict(cols=0)):    # nothing to do
        x0 = _logits(d_logits=None, **shape)
        assert _list(x0, None, 4, None, None, None) == odb.ODB_OK
        assert _list_back(x0, None, 4, None, None, None, None) == odb.ODB_OK
        assert _list(x0, None, 0, None, None, None) == BAD


def test_binding_refuses_other_shapes():
    import torch

    z = torch.zeros(2, 3, 10)
    ids = torch.zeros(2, 3, 4, dtype=torch.int32)
    out = torch.zeros(2, 3, 4)
    for bad in (ids[0], ids[:1], ids[:, :2], ids.view(6, 4), ids.long()):
        with pytest.raises(ValueError):
            odb.odb_token_list_logprobs(z, bad, out)
    with pytest.raises(ValueError):        # host tensors
        odb.odb_token_list_logprobs(z, ids, out)
    with pytest.raises(ValueError):
        odb.odb_token_list_logprobs_backward(z, ids, torch.zeros(2, 3, 2), out, torch.zeros(2, 3, 11))


def test_reference_gradient_is_the_slope():
    rng = np.random.default_rng(3)
    z = rng.standard_normal((2, 3, 9))
    y = rng.integers(0, 9, (2, 3)).astype(np.int32)
    y[0, 1] = -100
    ids = rng.integers(0, 9, (2, 3, 4)).astype(np.int32)
    ids[1, 2, 1] = -100
    g = rng.standard_normal((2, 3, 4))
    value = lambda x: float((ref.list_logprobs(x, y, ids, 1, 1.3)[0] * g).sum())
    grad = ref.list_logprobs_grad(z, y, ids, 1, 1.3, g)
    for at in np.ndindex(z.shape):
        up, down = z.copy(), z.copy()
        up[at] += 1e-5
        down[at] -= 1e-5
        assert abs((value(up) - value(down)) / 2e-5 - grad[at]) < 1e-7


def _top(x=None, labels=P, k=4, ids=P, top=P, logprob=P, rank=P, stats=P, entropy=P, ws=P, ws_bytes=1 << 40):
    return odb.load().odb_token_top_logprobs(byref(_logits() if x is None else x), labels, k, ids, top, logprob, rank,
                                             stats, entropy, None, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_LOGITS, ids=str)
def test_top_logits_refused(bad):
    assert _top(_logits(**bad)) == BAD and odb.load().odb_last_error_message() != b""


def test_top_arguments_refused():
    lib = odb.load()
    assert lib.odb_token_top_logprobs(None, P, 4, P, P, P, P, P, P, None, P, 1 << 40, None) == BAD
    for bad in (dict(k=0), dict(k=-3), dict(k=odb.ODB_LIST_MAX + 1), dict(ids=None), dict(top=None), dict(stats=P + 4),
                dict(labels=None), dict(labels=None, rank=None), dict(labels=None, logprob=None), dict(ws=None),
                dict(ws=P + 128)):
        assert _top(**bad) == BAD, bad
    x = _logits()
    size = lib.odb_token_top_workspace_size(byref(x), 4)
    assert size > 0
    assert _top(ws_bytes=size - 1) == odb.ODB_E_WORKSPACE
    for shape in (dict(rows=0), dict(cols=0)):
        x0 = _logits(d_logits=None, **shape)
        assert _top(x0, None, 4, None, None, None, None, None, None, None, 0) == odb.ODB_OK
    assert lib.odb_token_top_workspace_size(None, 4) == 0
    for k in (0, odb.ODB_LIST_MAX + 1):
        assert lib.odb_token_top_workspace_size(byref(x), k) == 0
    for bad in (dict(dtype=3), dict(vocab=0), dict(rows=-1), dict(rows=1 << 16, cols=1 << 15)):
        assert lib.odb_token_top_workspace_size(byref(_logits(**bad)), 4) == 0


def test_top_binding_refuses():
    import torch

    z = torch.zeros(2, 3, 10)
    ids, top = torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, 4)
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError):        # host tensors
        odb.odb_token_top_logprobs(z, ids, top, ws)
    with pytest.raises(ValueError):
        odb.odb_token_top_logprobs(z, ids[0], top, ws)


def test_reference_of_ties():
    row = np.array([1.0, 3.0, -np.inf, 3.0, 1.0, 0.0])
    assert ref.top(row, 4).tolist() == [1, 3, 0, 4] and ref.top(row, 9).tolist() == [1, 3, 0, 4, 5]
    assert [ref.rank(row, y) for y in range(6)] == [2, 0, 5, 1, 3, 4]


def _tiles(**kw):
    from test_losses_host import _tiles as tiles
    return tiles(**kw)


def _distill(t=None, p=None, k=4, student=P, teacher=P, w=None, loss=P, mean=P, count=P, grad=P, ws=P, ws_bytes=1 << 40):
    return odb.load().odb_distill_loss(byref(t or _tiles()), byref(p or odb.DistillParams()), k, student, teacher, w, loss,
                                       mean, count, grad, None, ws, ws_bytes, None)


def test_distill_arguments_refused():
    from test_losses_host import BAD_ARRAYS, BAD_TILES
    lib = odb.load()
    for bad in BAD_TILES + [dict(num_elems=(1 << 32) + 1)]:
        assert _distill(_tiles(**bad)) == BAD, bad
        assert lib.odb_distill_workspace_size(byref(_tiles(**bad)), 4) == 0
    for bad in BAD_ARRAYS:
        assert _distill(_tiles(**bad)) == BAD, bad
    for bad in (dict(kind=3), dict(kind=-1), dict(support=3), dict(support=-1), dict(reduce=3), dict(reduce=-1),
                dict(reserved0=1), dict(kind=2, mix=0.0), dict(kind=2, mix=1.0), dict(kind=2, mix=float("nan")),
                dict(kind=2, mix=1e-60), dict(kind=2, mix=1e-40), dict(kind=2, mix=-0.5), dict(loss_scale=float("inf")),
                dict(loss_scale=float("nan"))):
        assert _distill(p=odb.DistillParams(**bad)) == BAD, bad
    for bad in (dict(k=0), dict(k=odb.ODB_LIST_MAX + 1), dict(student=None), dict(teacher=None), dict(loss=None),
                dict(mean=None), dict(count=None), dict(ws=None), dict(ws=P + 8)):
        assert _distill(**bad) == BAD, bad
    size = lib.odb_distill_workspace_size(byref(_tiles()), 4)
    assert size > 0 and _distill(ws_bytes=size - 1) == odb.ODB_E_WORKSPACE
    for k in (0, odb.ODB_LIST_MAX + 1):
        assert lib.odb_distill_workspace_size(byref(_tiles()), k) == 0
    assert lib.odb_distill_workspace_size(None, 4) == 0
    # no slots: nothing to do
    assert _distill(_tiles(num_slots=0), loss=None, mean=None, count=None, student=None, ws=None) == odb.ODB_OK
    # a workspace grows with the run
    sizes = [lib.odb_distill_workspace_size(byref(_tiles(num_elems=n)), 4) for n in (50, 1 << 20, 1 << 32)]
    assert sizes[0] < sizes[1] < sizes[2]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("support", [0, 1, 2])
def test_reference_divergence_is_one(kind, support):
    """Against the definition in probabilities, its slopes against differences; 0 and flat where both agree."""
    rng = np.random.default_rng(kind * 3 + support)
    w = 0.3
    for _ in range(20):
        t = np.log(rng.dirichlet(np.ones(7))[:6] * 0.98)
        s = np.log(rng.dirichlet(np.ones(7))[:6] * 0.98)
        t[rng.integers(6)] = -np.inf
        on = t > -np.inf

        def value(s):
            p, q = np.exp(t[on]), np.exp(s[on])
            if support == 1:
                p, q = p / p.sum(), q / q.sum()
            elif support == 2:
                p, q = np.append(p, 1 - p.sum()), np.append(q, 1 - q.sum())
            kl = lambda a, b: float((a * np.log(a / b)).sum())
            m = w * p + (1 - w) * q
            return [kl(p, q), kl(q, p), w * kl(p, m) + (1 - w) * kl(q, m)][kind]

        v, g, _, _ = ref.distill_token(t, s, kind, support, w)
        assert abs(v - value(s)) < 1e-12
        for j in range(6):
            up, down = s.copy(), s.copy()
            up[j] += 1e-6
            down[j] -= 1e-6
            assert abs((value(up) - value(down)) / 2e-6 - g[j]) < 1e-7
        if support:
            v, g, _, _ = ref.distill_token(t, np.where(on, t, 0.0), kind, support, w)
            assert abs(v) < 1e-12 and np.abs(g).max() < 1e-12
