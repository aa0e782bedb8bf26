"""The operators over lists of tokens on the GPU against their definitions in 64 bits: types, strides, lists that
end early or name a token twice, masks that leave a row empty, infinities and NaN in places that do not count.

Tolerances count roundings of fp32 (U = 2^-24 relative each) and of the output's type."""
import math

import numpy as np
import pytest

import _lists as ref
from _losses import IGNORE, U
from _parity import log

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _types():
    torch = _torch()
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _dev(v):
    return None if v is None else _torch().from_numpy(np.ascontiguousarray(v)).cuda()


def _tile(rng, rows, cols, V, dtype, shift, pad, labels=True, masked=True):
    """Logits [rows, cols, V] (a view with a padded stride) on the GPU and in 64 bits with 0 where no token is
    scored, labels (or None), and which logits positions score a token."""
    torch = _torch()
    z = torch.from_numpy((rng.standard_normal((rows, cols, V)) * 2.5).astype(np.float32)).to(_types()[dtype])
    if masked and V > 40:
        z[:, :, 3::29] = -math.inf
        z[:, :, 5::31] = torch.finfo(z.dtype).min
    y = None
    if labels:
        y = rng.integers(0, V, (rows, cols)).astype(np.int32)
        if masked and V > 40:
            y[(y % 29 == 3) | (y % 31 == 5)] = 0
        y[rng.random((rows, cols)) < 0.25] = IGNORE
        if rows > 1:
            y[1] = IGNORE           # a row in which nothing counts
    on = ref.counted(y, rows, cols, V, shift)
    scored = np.zeros((rows, cols), bool)
    scored[:, :cols - shift] = on[:, shift:]
    z[torch.from_numpy(~scored)] = math.nan     # what does not count may hold anything
    wide = torch.full((rows, cols, V + pad), math.nan, dtype=z.dtype)
    wide[:, :, :V] = z
    z64 = np.where(scored[:, :, None], z.double().numpy(), 0.0)
    return wide.cuda()[:, :, :V], z64, y, on, scored


def _ids(rng, on, V, k):
    """Lists: some end early, some name a token twice, some are empty; anything where a token does not count."""
    ids = rng.integers(0, V, (*on.shape, k)).astype(np.int32)
    ids[rng.random(ids.shape) < 0.15] = IGNORE
    if k > 1:
        twice = rng.random(on.shape) < 0.3
        ids[twice, k - 1] = ids[twice, 0]
        ids[twice, k // 2] = ids[twice, 0]
    ids[rng.random(on.shape) < 0.1] = IGNORE
    ids[~on] = V + 12345
    return ids


LIST_CASES = [
    # rows, cols, V, dtype, shift, scale, pad, k, labels
    (1, 1, 1, "fp32", 0, 1.0, 0, 1, False), (1, 1, 7, "bf16", 0, 1.0, 0, 128, True), (2, 1, 64, "fp16", 1, 1.0, 0, 3, True),
    (3, 5, 63, "bf16", 1, 1.0, 0, 8, True), (2, 9, 257, "fp16", 1, 0.5, 3, 17, False),
    (4, 33, 65, "fp32", 1, 2.0, 1, 128, True), (3, 17, 1000, "fp16", 1, 1.0, 0, 5, True),
    (2, 8, 2049, "fp32", 1, 1.0, 0, 64, False), (2, 7, 4099, "bf16", 1, 1.0, 5, 127, True),
    (1, 6, 8191, "fp16", 1, 1.0, 0, 32, True), (2, 3, 32000, "fp32", 1, 1.0, 0, 2, True),
    (2, 4, 50021, "bf16", 1, 1.5, 11, 64, True), (1, 2, 151936, "bf16", 0, 1.0, 0, 128, False),
    (300, 3, 5, "bf16", 1, 1.0, 0, 4, True), (600, 2, 515, "bf16", 1, 0.8, 1, 9, True),
    (300, 2, 1030, "fp16", 0, 1.0, 0, 16, True), (270, 2, 5003, "bf16", 0, 1.0, 3, 20, True),
]


@pytest.mark.parametrize("case", LIST_CASES, ids=str)
def test_list_logprobs_and_gradient(case):
    import paper_2606_19989_amd as odb
    torch = _torch()
    rows, cols, V, dtype, shift, scale, pad, k, labels = case
    log(f"list logprobs {case}")
    rng = np.random.default_rng(rows * 1000 + cols * 10 + V + k)
    zd, z64, y, on, scored = _tile(rng, rows, cols, V, dtype, shift, pad, labels)
    ids = _ids(rng, on, V, k)
    want, stats = ref.list_logprobs(z64, y, ids, shift, scale)
    out = torch.full((rows, cols, k), 7.0, device="cuda")
    st = torch.full((rows, cols, 2), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    odb.odb_token_list_logprobs(zd, _dev(ids), out, labels=_dev(y), stats=st, status=status, shift=shift, scale=scale)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    got, gst = out.double().cpu().numpy(), st.double().cpu().numpy()
    assert np.all(gst[..., 0] == stats[..., 0])
    assert np.all(got[~on] == 0) and np.all(gst[~on] == 0)
    elt = 4 if dtype == "fp32" else 2
    e_lse = np.zeros((rows, cols))
    for i, c in zip(*np.nonzero(on)):
        row, L = z64[i, c - shift], stats[i, c, 1]
        e_lse[i, c] = ref.sum_bounds(V, elt, ref.spread(row, scale), L)
        assert abs(gst[i, c, 1] - L) <= e_lse[i, c]
        w, g = want[i, c], got[i, c]
        low = w < -3e38        # fp32's lowest times a scale: either side of the largest number
        assert np.all((g[low] < -3e38))
        w, g = w[~low], g[~low]
        assert np.all(np.abs(g - w) <= e_lse[i, c] + 2 * U * (np.abs(w) + abs(L)) + 3 * U * np.abs(w + L))

    g = rng.standard_normal((rows, cols, k)).astype(np.float32)
    g[rng.random((rows, cols, k)) < 0.1] = 0.0
    g[rng.random((rows, cols)) < 0.15] = 0.0       # a gradient of 0
    gin = g.copy()
    gin[~on] = math.nan                            # not read where nothing counts, nor where there is no entry
    gin[ids == IGNORE] = math.nan
    want = ref.list_logprobs_grad(z64, y, ids, shift, scale, g.astype(np.float64))
    back = torch.full((rows, cols, V + pad), 9.0, dtype=zd.dtype, device="cuda")
    odb.odb_token_list_logprobs_backward(zd, _dev(ids), st, _dev(gin), back[:, :, :V], labels=_dev(y), status=status,
                                         shift=shift, scale=scale)
    got = back.double().cpu().numpy()
    assert int(status.item()) == 0
    assert np.all(got[:, :, V:] == 9.0), "written beyond the vocabulary"
    got = got[:, :, :V]
    assert np.all(got[~scored] == 0)
    fin = torch.finfo(zd.dtype)
    for i, c in zip(*np.nonzero(scored)):
        at = (i, c + shift)
        real = ids[at] != IGNORE
        gs, vs = np.abs(g[at][real].astype(np.float64)), ids[at][real]
        x = scale * (z64[i, c] - z64[i, c].max())
        p = np.exp(x - stats[at][1])
        x = np.abs(np.where(p > 0, x, 0.0))
        G = gs.sum()
        tol = p * G * (U * (3 * x + 16 + k) + e_lse[at])
        at_ids = np.zeros(V)
        np.add.at(at_ids, vs, gs)
        tol = scale * (tol + at_ids * U * (k + 4))
        tol += (fin.eps / 2) * np.abs(want[i, c]) * (1 + 1e-3) + float(fin.smallest_normal) * fin.eps / 2
        err = np.abs(got[i, c] - want[i, c])
        assert np.all(err <= tol), (i, c, err.max(), (err / tol).max())
    # in place, the same bit for bit
    odb.odb_token_list_logprobs_backward(zd, _dev(ids), st, _dev(gin), zd, labels=_dev(y), status=status, shift=shift,
                                         scale=scale)
    assert torch.equal(zd, back[:, :, :V])


def test_list_of_the_label_is_the_label():
    """A list of one entry, the label: odb_token_logprobs' numbers and gradient."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(5)
    zd, z64, y, on, _ = _tile(rng, 4, 21, 3001, "bf16", 1, 5)
    yd = _dev(y)
    a, sa, b, sb = (torch.empty(4, 21, n, device="cuda") for n in (1, 2, 1, 2))
    odb.odb_token_logprobs(zd, yd, a, stats=sa)
    odb.odb_token_list_logprobs(zd, yd.view(4, 21, 1), b, labels=yd, stats=sb)
    assert torch.equal(sa, sb) and torch.equal(a, b)
    g = torch.randn(4, 21, device="cuda")
    ga, gb = torch.empty_like(zd), torch.empty_like(zd)
    odb.odb_token_logprobs_backward(zd, yd, sa, g, ga)
    odb.odb_token_list_logprobs_backward(zd, yd.view(4, 21, 1), sa, g.view(4, 21, 1), gb, labels=yd)
    # p (1 - p) in one rounding more or less, then bf16's
    err = (ga.double() - gb.double()).abs()
    assert bool((err <= 2.0 ** -7 * ga.double().abs() + 8 * U * g.abs().max().double()).all())


def test_bad_ids_are_reported_and_no_entries():
    import paper_2606_19989_amd as odb
    torch = _torch()
    z = torch.randn(1, 2, 50, device="cuda")
    ids = torch.tensor([[[3, 50, -1], [2, IGNORE, 7]]], dtype=torch.int32, device="cuda")
    out, st = torch.empty(1, 2, 3, device="cuda"), torch.empty(1, 2, 2, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    odb.odb_token_list_logprobs(z, ids, out, stats=st, status=status, shift=0)
    assert int(status.item()) != 0
    lp = torch.log_softmax(z.double(), -1)
    want = torch.tensor([[lp[0, 0, 3], 0, 0], [lp[0, 1, 2], 0, lp[0, 1, 7]]], device="cuda")
    assert float((out[0].double() - want).abs().max()) < 1e-5 and bool((out[0][want == 0] == 0).all())
    status.zero_()
    g = torch.ones(1, 2, 3, device="cuda")
    back = torch.empty_like(z)
    odb.odb_token_list_logprobs_backward(z, ids, st, g, back, status=status, shift=0)
    assert int(status.item()) != 0
    g2 = g.clone()
    g2[0, 0, 1:] = 0
    ids2 = ids.clone()
    ids2[0, 0, 1:] = IGNORE
    again = torch.empty_like(z)
    status.zero_()
    odb.odb_token_list_logprobs_backward(z, ids2, st, g2, again, status=status, shift=0)
    assert int(status.item()) == 0 and torch.equal(back, again)


@pytest.mark.parametrize("bad", ["nan", "inf", "all -inf"])
def test_logits_without_a_distribution(bad):
    import paper_2606_19989_amd as odb
    torch = _torch()
    z = torch.randn(2, 1, 1000, device="cuda", dtype=torch.bfloat16)
    if bad == "all -inf":
        z[0] = -math.inf
    else:
        z[0, 0, 777] = float(bad)
    ids = torch.tensor([[[0, 777, IGNORE]], [[0, 777, IGNORE]]], dtype=torch.int32, device="cuda")
    out, st = torch.empty(2, 1, 3, device="cuda"), torch.empty(2, 1, 2, device="cuda")
    odb.odb_token_list_logprobs(z, ids, out, stats=st, shift=0)
    assert bool(out[0, 0, :2].isnan().all()) and float(out[0, 0, 2]) == 0
    assert bool(out[1].isfinite().all())


def test_a_listed_token_at_minus_infinity():
    import paper_2606_19989_amd as odb
    torch = _torch()
    z = torch.randn(1, 1, 300, device="cuda")
    z[0, 0, 9] = -math.inf
    ids = torch.tensor([[[9, 10]]], dtype=torch.int32, device="cuda")
    out, st = torch.empty(1, 1, 2, device="cuda"), torch.empty(1, 1, 2, device="cuda")
    odb.odb_token_list_logprobs(z, ids, out, stats=st, shift=0)
    assert float(out[0, 0, 0]) == -math.inf and math.isfinite(float(out[0, 0, 1]))
    g = torch.tensor([[[0.5, -0.25]]], device="cuda")
    back = torch.empty_like(z)
    odb.odb_token_list_logprobs_backward(z, ids, st, g, back, shift=0)
    assert float(back[0, 0, 9]) == 0.5 and bool(back.isfinite().all())


def test_gradient_against_differences():
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(17)
    z = torch.from_numpy(rng.standard_normal((1, 3, 40)).astype(np.float32)).cuda()
    ids = torch.from_numpy(rng.integers(0, 40, (1, 3, 6)).astype(np.int32)).cuda()
    ids[0, 1, 4] = ids[0, 1, 2]
    g = torch.from_numpy(rng.standard_normal((1, 3, 6)).astype(np.float32)).cuda()

    def value(x):
        out, st = torch.empty(1, 3, 6, device="cuda"), torch.empty(1, 3, 2, device="cuda")
        odb.odb_token_list_logprobs(x, ids, out, stats=st, shift=0, scale=1.5)
        return float((out.double() * g.double()).sum()), st

    _, st = value(z)
    back = torch.empty_like(z)
    odb.odb_token_list_logprobs_backward(z, ids, st, g, back, shift=0, scale=1.5)
    h = 2.0 ** -7
    for c, v in [(0, 0), (0, int(ids[0, 0, 0])), (1, int(ids[0, 1, 2])), (2, 39)]:
        up, down = z.clone(), z.clone()
        up[0, c, v] += h
        down[0, c, v] -= h
        slope = (value(up)[0] - value(down)[0]) / (float(up[0, c, v]) - float(down[0, c, v]))
        # the third derivative is below 6 * 1.5^3 * sum |g|; values of 18 entries of about 5 are right to U each
        most = float(g.abs().sum())
        assert abs(slope - float(back[0, c, v])) <= h * h * 1.5 ** 3 * most + 16 * U * 6 * most / h
