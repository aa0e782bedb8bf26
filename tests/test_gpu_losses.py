"""The loss operators on the GPU against their definitions in 64 bits: types, strides, masks that
leave a row empty, infinities and NaN in places that do not count, slots and rows across chunk
ends, pairs spread over tiles, other streams, graphs, and the whole chain behind a collate.

Tolerances count roundings of fp32 (U = 2^-24 relative each) and of the output's type."""
import math

import numpy as np
import pytest

import _losses as ref
import synth
from _losses import IGNORE, U, Plan
from _parity import log

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _types():
    torch = _torch()
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _logprob_bounds(V, L, x, second, ent):
    """Absolute error bounds of logsum, logprob and entropy.  A thread adds at most V / 64 terms
    (V / 256 above 2,048) and joins eight levels; every rescaling and every term's exponent and
    power add (3 |x| + 3) U, and sum p |x| <= sqrt(sum p x^2)."""
    adds = V / (64 if V <= 2048 else 256) + 32
    root = np.sqrt(second)
    lse = U * (adds + 8 + 3 * root + 2 * np.abs(L))
    lp = lse + U * (3 * x + 2 * (x + np.abs(L)))
    # entropy = logsum - t / s: t is a sum of terms of magnitude p |x| with the same roundings
    en = lse + U * (2 * (adds + 8) * (root + 1) + 6 * second + 2 * np.abs(L) + 2 * np.abs(ent))
    return lse, lp, en


def _logits(rng, rows, cols, V, dtype, spread=2.5):
    torch = _torch()
    return torch.from_numpy((rng.standard_normal((rows, cols, V)) * spread).astype(np.float32)).to(_types()[dtype])


LOGPROB_CASES = [
    # rows, cols, V, dtype, shift, scale, pad, entropy
    (1, 1, 1, "fp32", 0, 1.0, 0, True), (1, 1, 7, "bf16", 0, 1.0, 0, False), (2, 1, 64, "fp16", 1, 1.0, 0, True),
    (3, 5, 63, "bf16", 1, 1.0, 0, True), (2, 9, 257, "fp16", 1, 0.5, 3, True), (4, 33, 65, "fp32", 1, 2.0, 1, True),
    (3, 17, 1000, "fp16", 1, 1.0, 0, False), (2, 8, 2047, "bf16", 0, 1.25, 0, True),
    (2, 8, 2048, "bf16", 1, 1.0, 8, False), (2, 8, 2049, "fp32", 1, 1.0, 0, True),
    (2, 7, 4099, "bf16", 1, 1.0, 5, True), (1, 6, 8191, "fp16", 1, 1.0, 0, True),
    (1, 5, 8192, "bf16", 0, 0.75, 0, False), (2, 3, 32000, "fp32", 1, 1.0, 0, True),
    (2, 4, 50021, "bf16", 1, 1.5, 11, True), (1, 3, 50021, "fp16", 1, 1.0, 1, False),
    (1, 3, 151936, "bf16", 1, 1.0, 0, True), (300, 3, 5, "bf16", 1, 1.0, 0, True),
]


@pytest.mark.parametrize("case", LOGPROB_CASES, ids=str)
def test_token_logprobs_and_gradient(case):
    import paper_2606_19989_amd as odb
    torch = _torch()
    rows, cols, V, dtype, shift, scale, pad, entropy = case
    log(f"token logprobs {case}")
    rng = np.random.default_rng(rows * 1000 + cols * 10 + V)
    wide = torch.full((rows, cols, V + pad), math.nan, dtype=_types()[dtype])
    z = _logits(rng, rows, cols, V, dtype)
    if V > 40:      # masked vocabulary entries
        z[:, :, 3::29] = -math.inf
        z[:, :, 5::31] = torch.finfo(z.dtype).min
    y = rng.integers(0, V, (rows, cols)).astype(np.int32)
    if V > 40:
        y[(y % 29 == 3) | (y % 31 == 5)] = 0
    y[rng.random((rows, cols)) < 0.25] = IGNORE
    if rows > 1:
        y[1] = IGNORE           # a row in which nothing counts
    on = y != IGNORE
    on[:, :shift] = False
    scored = np.zeros((rows, cols), bool)       # logits positions that score a token
    scored[:, :cols - shift] = on[:, shift:]
    z[torch.from_numpy(~scored)] = math.nan     # what does not count may hold anything
    wide[:, :, :V] = z
    zd = wide.cuda()[:, :, :V]
    yd = torch.from_numpy(y).cuda()
    z64 = np.where(scored[:, :, None], z.double().numpy(), 0.0)
    lp, stats, ent, second, at = ref.token_logprobs(z64, y, shift, scale)
    out = [torch.full((rows, cols), 7.0, device="cuda") for _ in range(2)] + [
        torch.full((rows, cols, 2), 7.0, device="cuda")]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    odb.odb_token_logprobs(zd, yd, out[0], stats=out[2], entropy=out[1] if entropy else None, status=status,
                           shift=shift, scale=scale)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    g_lp, g_ent, g_stats = (o.double().cpu().numpy() for o in out)
    e_lse, e_lp, e_ent = _logprob_bounds(V, stats[..., 1], at, second, ent)
    assert np.all(g_stats[..., 0] == stats[..., 0])
    assert np.all(np.abs(g_stats[..., 1] - stats[..., 1]) <= e_lse)
    assert np.all(np.abs(g_lp - lp) <= e_lp)
    assert np.all(g_lp[~on] == 0) and np.all(g_stats[~on] == 0)
    if entropy:
        assert np.all(np.abs(g_ent - ent) <= e_ent)
        assert np.all(g_ent[~on] == 0)

    # the gradient
    g = rng.standard_normal((rows, cols)).astype(np.float32)
    h = (rng.standard_normal((rows, cols)) * 0.3).astype(np.float32) if entropy else None
    zero = rng.random((rows, cols)) < 0.2
    g[zero] = 0.0
    if entropy:
        h[zero & (rng.random((rows, cols)) < 0.5)] = 0.0
    gin, hin = g.copy(), None if h is None else h.copy()
    gin[~on] = math.nan          # not read where nothing counts
    if hin is not None:
        hin[~on] = math.nan
    want = ref.token_logprobs_grad(z64, y, shift, scale, np.where(on, g, 0.0).astype(np.float64),
                                   None if h is None else np.where(on, h, 0.0).astype(np.float64))
    back = torch.full((rows, cols, V + pad), 9.0, dtype=z.dtype, device="cuda")
    dev = lambda v: None if v is None else torch.from_numpy(v).cuda()
    odb.odb_token_logprobs_backward(zd, yd, out[2], dev(gin), back[:, :, :V],
                                    entropy=out[1] if entropy else None, grad_entropy=dev(hin), status=status,
                                    shift=shift, scale=scale)
    got = back.double().cpu().numpy()
    assert np.all(got[:, :, V:] == 9.0), "written beyond the vocabulary"
    got = got[:, :, :V]
    assert np.all(got[~scored] == 0)
    fin = torch.finfo(z.dtype)
    for i, c in zip(*np.nonzero(scored)):
        t = (i, c + shift)
        x = scale * (z64[i, c] - z64[i, c].max())
        p = np.exp(x - stats[t][1])
        x = np.maximum(np.abs(np.where(p > 0, x, 0.0)), 0.0)
        ag, ah = abs(scale * g[t]), abs(scale * h[t]) if entropy else 0.0
        mag = ag + ah * (abs(stats[t][1]) + abs(ent[t]) + x)
        tol = p * mag * (U * (3 * x + 16) + e_lse[t]) + p * ah * (e_ent[t] + 2 * e_lse[t]) + 2.0 ** -126 * mag
        tol[y[t]] += 4 * U * ag
        tol += (fin.eps / 2) * np.abs(want[i, c]) * (1 + 1e-3) + float(fin.smallest_normal) * fin.eps / 2
        err = np.abs(got[i, c] - want[i, c])
        assert np.all(err <= tol), (i, c, err.max(), (err / tol).max())
    # in place
    odb.odb_token_logprobs_backward(zd, yd, out[2], dev(gin), zd, entropy=out[1] if entropy else None,
                                    grad_entropy=dev(hin), shift=shift, scale=scale)
    assert torch.equal(zd, back[:, :, :V])


def test_gradient_with_another_alignment_than_the_logits():
    """Logits rows and gradient rows that start at different offsets from 16 bytes."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(8)
    for dtype in ("bf16", "fp32"):
        for a, b in ((0, 1), (1, 0), (3, 2), (1, 4)):
            z = _logits(rng, 2, 5, 4097, dtype).cuda()
            buf = torch.empty(2 * 5 * 4110 + 8, dtype=z.dtype, device="cuda")
            zd = buf[a:a + 2 * 5 * 4110].view(2, 5, 4110)[:, :, :4097]
            zd.copy_(z)
            y = torch.from_numpy(rng.integers(0, 4097, (2, 5)).astype(np.int32)).cuda()
            lp, st = torch.empty(2, 5, device="cuda"), torch.empty(2, 5, 2, device="cuda")
            lp2, st2 = torch.empty_like(lp), torch.empty_like(st)
            odb.odb_token_logprobs(z, y, lp, stats=st)
            odb.odb_token_logprobs(zd, y, lp2, stats=st2)
            assert torch.equal(lp, lp2) and torch.equal(st, st2)
            g = torch.randn(2, 5, device="cuda")
            want, out = torch.empty_like(z), torch.empty(2 * 5 * 4099 + 8, dtype=z.dtype, device="cuda").fill_(5.0)
            od = out[b:b + 2 * 5 * 4099].view(2, 5, 4099)[:, :, :4097]
            odb.odb_token_logprobs_backward(z, y, st, g, want)
            odb.odb_token_logprobs_backward(zd, y, st, g, od)
            assert torch.equal(od, want), (dtype, a, b)
            assert torch.all(out[:b] == 5) and torch.all(out[b + 2 * 5 * 4099:] == 5)
            assert torch.all(out[b:b + 2 * 5 * 4099].view(2, 5, 4099)[:, :, 4097:] == 5)


def test_rows_without_a_distribution_and_masked_labels():
    import paper_2606_19989_amd as odb
    torch = _torch()
    inf = math.inf
    for V in (16, 5000):
        for dtype in ("fp32", "bf16", "fp16"):
            t = _types()[dtype]
            z = torch.zeros(1, 7, V, dtype=t)
            z[0, 0] = torch.finfo(t).min             # all the type's lowest: uniform
            z[0, 1] = -inf                           # no distribution
            z[0, 2, 1] = inf
            z[0, 3, 2] = math.nan
            z[0, 4, 3] = -inf                        # the label itself masked
            z[0, 5, 1:] = -inf                       # one entry left
            z[0, 6, 1:] = torch.finfo(t).min
            y = torch.tensor([[1, 0, 1, 0, 3, 0, 0]], dtype=torch.int32)
            lp, st, H = (torch.empty(1, 7, device="cuda"), torch.empty(1, 7, 2, device="cuda"),
                         torch.empty(1, 7, device="cuda"))
            zd, yd = z.cuda(), y.cuda()
            odb.odb_token_logprobs(zd, yd, lp, stats=st, entropy=H, shift=0)
            v, e = lp.cpu()[0], H.cpu()[0]
            # V terms of 1 each: their sum is exact, its logarithm off by at most one rounding and a half
            assert abs(float(v[0]) + math.log(V)) <= 3 * U * math.log(V)
            assert abs(float(e[0]) - math.log(V)) <= 3 * U * math.log(V)
            assert all(math.isnan(float(v[i])) and math.isnan(float(e[i])) for i in (1, 2, 3))
            assert float(v[4]) == -inf and abs(float(e[4]) - math.log(V - 1)) <= 3 * U * math.log(V)
            assert float(v[5]) == 0 and float(e[5]) == 0 and float(v[6]) == 0 and float(e[6]) == 0
            g = torch.ones(1, 7, device="cuda")
            out = torch.empty_like(zd)
            odb.odb_token_logprobs_backward(zd, yd, st, g, out, shift=0)
            o = out.double().cpu()[0]
            rel = torch.finfo(t).eps / 2 + 8 * U * math.log(V)
            assert abs(float(o[0, 1]) - (1 - 1 / V)) <= rel
            assert torch.all((o[0, 2:] + 1 / V).abs() <= rel / V)
            for i in (1, 2, 3):
                assert torch.isnan(o[i]).any()
            assert float(o[4, 3]) == 1.0 and torch.all(o[5] == 0) and torch.all(o[6] == 0)
            # a token whose gradient is 0 is not read
            odb.odb_token_logprobs_backward(zd, yd, st, torch.zeros_like(g), out, shift=0)
            assert torch.all(out == 0)


def test_bad_labels_are_reported_and_do_not_count():
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(4)
    for V in (50, 3000):
        z = _logits(rng, 2, 4, V, "bf16").cuda()
        y = torch.tensor([[1, V, 2, 3], [0, 5, -1, -2 ** 31]], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        lp, st = torch.empty(2, 4, device="cuda"), torch.empty(2, 4, 2, device="cuda")
        odb.odb_token_logprobs(z, y, lp, stats=st, status=status)
        assert int(status.item()) != 0
        on = torch.tensor([[0, 0, 1, 1], [0, 1, 0, 0]], dtype=torch.bool)
        assert torch.equal(lp.cpu() != 0, on)
        status.zero_()
        out = torch.empty_like(z)
        odb.odb_token_logprobs_backward(z, y, st, torch.ones(2, 4, device="cuda"), out, status=status)
        assert int(status.item()) != 0
        assert torch.equal((out != 0).any(-1).cpu()[:, :3], on[:, 1:])
        odb.odb_token_logprobs(z, y, lp)     # without a status word
        assert torch.equal(lp.cpu() != 0, on)


def test_other_orders_of_rows_and_columns():
    """Logits kept position first, and logits of one position broadcast over the tile."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(9)
    z = _logits(rng, 3, 6, 300, "bf16").cuda()
    y = torch.from_numpy(rng.integers(0, 300, (3, 6)).astype(np.int32)).cuda()
    a, b, st = torch.empty(3, 6, device="cuda"), torch.empty(3, 6, device="cuda"), torch.empty(3, 6, 2, device="cuda")
    odb.odb_token_logprobs(z, y, a, stats=st)
    first = z.transpose(0, 1).contiguous().transpose(0, 1)
    odb.odb_token_logprobs(first, y, b)
    assert torch.equal(a, b)
    g = torch.randn(3, 6, device="cuda")
    o1, o2 = torch.empty_like(z), torch.empty(6, 3, 300, dtype=z.dtype, device="cuda").transpose(0, 1)
    odb.odb_token_logprobs_backward(z, y, st, g, o1)
    odb.odb_token_logprobs_backward(first, y, st, g, o2)
    assert torch.equal(o1, o2)
    odb.odb_token_logprobs(z[:1, :1].expand(3, 6, 300), y, b, shift=0)
    odb.odb_token_logprobs(z[:1, :1].expand(3, 6, 300).contiguous(), y, a, shift=0)
    assert torch.equal(a, b)
    with pytest.raises(odb.OdbError):
        odb.odb_token_logprobs_backward(z, y, st, g, z[:1, :1].expand(3, 6, 300))


def test_more_positions_than_a_grid_holds():
    """34 M positions of five logits, more than 2^20 blocks take at once."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    n, V = 34_000_003, 5
    log(f"{n} positions")
    gen = torch.Generator("cuda").manual_seed(1)
    z = torch.randn(1, n, V, generator=gen, device="cuda").half()
    y = torch.randint(0, V, (1, n), generator=gen, device="cuda", dtype=torch.int32)
    y[0, ::7] = IGNORE
    lp, H = torch.empty(1, n, device="cuda"), torch.empty(1, n, device="cuda")
    st = torch.empty(1, n, 2, device="cuda")
    odb.odb_token_logprobs(z, y, lp, stats=st, entropy=H, shift=0)
    on = y[0] != IGNORE
    want = torch.log_softmax(z[0].double(), -1)
    at = want.gather(1, y[0].long().clamp(min=0)[:, None])[:, 0]
    # logits of at most 8: the sum of five powers, its logarithm and the difference, all of size 20 or less
    assert float((lp[0].double() - at)[on].abs().max()) <= 32 * 20 * U
    assert float(lp[0][~on].abs().max()) == 0.0
    want = want.exp_()
    del at
    dz = torch.empty_like(z)
    odb.odb_token_logprobs_backward(z, y, st, torch.ones_like(lp), dz, shift=0)
    want = -want
    want[on] += torch.nn.functional.one_hot(y[0][on].long(), V)
    want[~on] = 0.0
    # rounded to fp16 (2^-11 of at most 1), or to its smallest step
    assert float((dz[0].double() - want).abs().max()) <= 2.0 ** -11 + 64 * U
    assert float(dz[0][~on].abs().max()) == 0.0


def test_logits_past_32_bits():
    """A tile of more than 2^32 bytes (and 2^31 elements) of logits: the last rows are right."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rows, cols, V = 64, 168, 200003       # 2.15e9 elements
    log(f"logits past 32 bits: {rows} x {cols} x {V}")
    z = torch.empty(rows, cols, V, dtype=torch.bfloat16, device="cuda")
    for r in range(rows):
        z[r].normal_()
    y = torch.randint(0, V, (rows, cols), dtype=torch.int32, device="cuda")
    keep = torch.zeros(rows, cols, dtype=torch.bool, device="cuda")
    keep[0, 1], keep[rows - 1, cols - 1], keep[rows - 1, 5] = True, True, True
    y = torch.where(keep, y, torch.full_like(y, IGNORE))
    lp, st = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, 2, device="cuda")
    odb.odb_token_logprobs(z, y, lp, stats=st)
    g = torch.ones(rows, cols, device="cuda")
    want = {}
    for i, c in keep.nonzero().tolist():
        row = z[i, c - 1].double()
        want[i, c] = torch.log_softmax(row, -1)
        L = float(st[i, c, 1])
        assert abs(float(lp[i, c]) - float(want[i, c][y[i, c].long()])) <= U * (V / 256 + 100 + 4 * L)
    odb.odb_token_logprobs_backward(z, y, st, g, z)        # in place: no second buffer of 4 GB
    for (i, c), lq in want.items():
        d = -lq.exp()
        d[y[i, c].long()] += 1
        err = (z[i, c - 1].double() - d).abs()
        assert torch.all(err <= d.abs() * (2.0 ** -8 + U * (V / 256 + 200)) + 1e-30)
    scored = torch.zeros(rows, cols, dtype=torch.bool, device="cuda")
    scored[:, :-1] = keep[:, 1:]
    for r in (0, rows // 2, rows - 1):
        assert torch.all(z[r][~scored[r]] == 0)


# ------------------------------------------------------------------------- tiles
def _plans():
    rng = np.random.default_rng(21)
    long = [int(x) for x in rng.integers(900, 1300, 9)]
    return {
        "one_token": Plan([[1]]), "two_rows": Plan([[1, 3]]), "idle_only": Plan([[], []]),
        "small": Plan([[4, 6], [], [9]]), "ones": Plan([[1] * 700, [1]]), "twos": Plan([[1, 2] * 1300]),
        "threes": Plan([[3, 2, 5, 5]] * 40 + [[]] * 3 + [[5] * 33] * 50),
        "chunk": Plan([[4096]]), "chunk_and_one": Plan([[4097], [1]]), "half_chunks": Plan([[2048, 2048], [2048]]),
        "long_row": Plan([[9000]]), "long_rows": Plan([[5000, 8191], [13], [1025, 1024]]),
        "mixed": Plan([sorted(long), [17] * 64, [], [300, 301, 340], [33] * 120, [2, 2, 2]], base=(5, 1 << 33)),
        "groups": Plan([[int(x) for x in sorted(rng.integers(1, 64, 30))] for _ in range(25)], base=(1 << 20, 77)),
    }


def _tiles(plan, labels, shift, extra_rows=3, extra_elems=5):
    """Device tiles whose arrays are longer than the run (what lies behind must stay)."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    y = np.concatenate([labels, np.full(extra_elems, 1, np.int32)])
    return odb.Tiles(dev(plan.rows), dev(plan.maxlen), dev(plan.row_off), dev(plan.tile_off), dev(y),
                     plan.R + extra_rows, shift=shift)


def _pad(x, extra, fill=math.nan):
    return None if x is None else _torch().from_numpy(np.concatenate(
        [x, np.full((extra,) + x.shape[1:], fill, x.dtype)])).cuda()


def _inputs(plan, rng, on):
    """Log-probabilities with NaN and infinities wherever nothing counts."""
    def junk(x):
        x = x.astype(np.float32)
        x[~on] = rng.choice([math.nan, math.inf, -math.inf], (~on).sum())
        return x
    lp = -np.abs(rng.standard_normal(plan.E)) * 2
    return (junk(lp), junk(lp + rng.standard_normal(plan.E) * 0.25), junk(lp + rng.standard_normal(plan.E) * 0.7),
            junk(rng.random(plan.E) * 5))


POLICY_OPTIONS = [
    dict(kl=3, reduce=0), dict(kl=3, reduce=1), dict(kl=2, reduce=2, loss_scale=0.01), dict(kl=1, reduce=0, dual_clip=1.3),
    dict(kl=0, reduce=1, token_advantage=1), dict(kl=3, reduce=1, entropy_coef=0.02, dual_clip=2.0),
    dict(kl=0, reduce=0, clip_low=1.0, clip_high=math.inf), dict(kl=3, reduce=0, clip_low=0.0, clip_high=0.0, old=False),
    dict(kl=2, reduce=1, entropy_coef=-0.5, token_advantage=1, weight=False),
]


def _policy_run(tiles, plan, p, lp, old, kref, H, adv, w, extra=5, ws=None, stream=None, sentinel=-3.0):
    import paper_2606_19989_amd as odb
    torch = _torch()
    E = plan.E + extra
    f = lambda *s: torch.full(s, sentinel, device="cuda")
    out = dict(loss=f(plan.K), means=f(plan.K, 4), counts=torch.full((plan.K, 4), -3, dtype=torch.int64, device="cuda"),
               grad=f(E), grad_ent=f(E) if H is not None else None)
    ws = torch.full((odb.odb_loss_workspace_size(tiles),), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    odb.odb_policy_loss(tiles, odb.PolicyParams(**p), lp, adv, out["loss"], out["means"], out["counts"], ws,
                        old_logprob=old, ref_logprob=kref, entropy=H, slot_weight=w, grad_logprob=out["grad"],
                        grad_entropy=out["grad_ent"], status=status, stream=stream)
    return out, status


def _policy_params(o):
    p = dict(kl=0, reduce=0, token_advantage=0, clip_low=0.2, clip_high=0.28, dual_clip=0.0, kl_coef=0.05,
             entropy_coef=0.0, loss_scale=4.0)
    p.update({k: v for k, v in o.items() if k in p})
    return p


@pytest.mark.parametrize("name", list(_plans()))
@pytest.mark.parametrize("shift", [0, 1])
def test_policy_loss(name, shift):
    torch = _torch()
    plan = _plans()[name]
    for n, o in enumerate(POLICY_OPTIONS):
        log(f"policy loss {name} shift={shift} {o}")
        rng = np.random.default_rng(100 + n)
        p = _policy_params(o)
        y = plan.labels(rng, 0.4, 0.1) if n % 3 else plan.labels(rng)
        if n == 3 and plan.K > 1:       # a slot in which nothing counts
            y[(plan.slot_of_row[plan.row_of] == plan.K - 1)] = IGNORE
        on = plan.counted(y, shift)
        lp, old, kref, H = _inputs(plan, rng, on)
        adv = rng.standard_normal(plan.E if p["token_advantage"] else plan.R).astype(np.float32)
        adv[rng.random(len(adv)) < 0.1] = 0.0
        old = old if o.get("old", True) else None
        kref = kref if p["kl"] else None
        H = H if p["entropy_coef"] else None
        w = rng.random(plan.K) if o.get("weight", True) else None
        want = ref.policy_loss(plan, y, shift, p, lp, old, kref, H, adv, w)
        tiles = _tiles(plan, y, shift)
        args = (_pad(lp, 5), _pad(old, 5), _pad(kref, 5), _pad(H, 5), _pad(adv, 5),
                None if w is None else torch.from_numpy(w).cuda())
        out, status = _policy_run(tiles, plan, p, *args)
        assert int(status.item()) == 0
        got = {k: v.double().cpu().numpy() for k, v in out.items() if v is not None}
        assert np.array_equal(got["counts"], want["counts"])
        far = 0.0 if old is None or not on.any() else np.abs(lp[on].astype(np.float64) - old[on]).max()
        # per token: the power and its argument, the series, products; a sum of such terms keeps the bound
        C = (80 + 2 * far) * U
        scale = p["loss_scale"] * (np.ones(plan.K) if w is None else w)
        mag = want["mags"][:, 0] + abs(p["kl_coef"]) * want["mags"][:, 1] + abs(p["entropy_coef"]) * want["mags"][:, 2]
        assert np.all(np.abs(got["loss"] - want["loss"]) <= C * scale * mag + 2 * U * np.abs(want["loss"]))
        assert np.all(np.abs(got["means"] - want["means"]) <= C * want["mags"])
        assert np.all(np.abs(got["grad"][:plan.E] - want["grad"]) <= 2 * C * want["grad_mag"])
        assert np.all(got["grad"][:plan.E][~on] == 0) and np.all(got["grad"][plan.E:] == -3.0)
        if H is not None:
            assert np.all(np.abs(got["grad_ent"][:plan.E] - want["grad_ent"]) <= 4 * U * np.abs(want["grad_ent"]))
            assert np.all(got["grad_ent"][plan.E:] == -3.0)
        again, _ = _policy_run(tiles, plan, p, *args)
        for k, v in out.items():
            assert v is None or torch.equal(v, again[k]), k


def test_fewer_than_four_elements():
    """Runs whose arrays end before a group of four does, at each of their addresses."""
    torch = _torch()
    for E in (1, 2, 3, 4, 5):
        for off in range(4):
            plan = Plan([[E]])
            rng = np.random.default_rng(E)
            y = plan.labels(rng)
            lp, old, kref, H = (v.astype(np.float32) for v in _inputs(plan, rng, y != IGNORE))
            adv = np.ones(1, np.float32)
            at = lambda v: torch.from_numpy(np.concatenate([np.zeros(off, v.dtype), v])).cuda()[off:]
            tiles = _tiles(plan, y, 0, 0, 0)
            for n, o in enumerate(POLICY_OPTIONS):
                p = _policy_params({**o, "token_advantage": 0})
                p["entropy_coef"] = 0.0
                want = ref.policy_loss(plan, y, 0, p, lp, old, kref, None, adv, None)
                out, status = _policy_run(tiles, plan, p, at(lp), at(old), at(kref), None, at(adv), None, extra=0)
                assert int(status.item()) == 0
                assert np.allclose(out["grad"].cpu().numpy(), want["grad"], rtol=200 * U, atol=1e-7)
            p = dict(kind=0, normalize=0, beta=1.0, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
            out, status = _preference_run(tiles, plan, p, at(lp), at(kref), None, torch.zeros(1, dtype=torch.int32,
                                                                                             device="cuda"), 0, 0)
            _check_preference(out, ref.preference_loss(plan, y, 0, p, lp, kref, None, np.zeros(1, np.int32)), plan, p,
                              lp, kref, y != IGNORE)


def test_policy_clips_are_decided_on_the_exact_difference():
    """Differences of one fp32 step around each bound, and equal to it."""
    torch = _torch()
    p = _policy_params(dict(dual_clip=1.5))
    bounds = [math.log1p(-0.2), math.log1p(0.28), math.log(1.5)]
    d = np.array([np.nextafter(np.float32(b), np.float32(s), dtype=np.float32) for b in bounds for s in (-9, b, 9)],
                 np.float32)
    lp = np.concatenate([d, d, d]).astype(np.float32)
    plan = Plan([[len(lp)]])
    y = np.ones(plan.E, np.int32)
    old = np.zeros_like(lp)
    adv = np.concatenate([np.full(9, 1.0), np.full(9, -1.0), np.zeros(9)]).astype(np.float32)
    p["token_advantage"] = 1
    want = ref.policy_loss(plan, y, 0, p, lp, old, None, None, adv, None)
    tiles = _tiles(plan, y, 0, 0, 0)
    dev = lambda x: torch.from_numpy(x).cuda()
    out, _ = _policy_run(tiles, plan, p, dev(lp), dev(old), None, None, dev(adv), None, extra=0)
    assert np.array_equal(out["counts"].cpu().numpy(), want["counts"])
    assert np.array_equal(out["grad"].cpu().numpy() == 0, want["grad"] == 0)
    # far ratios: a power that overflows fp32 where it is clipped, and where the advantage is 0
    lp = np.array([200.0, 200.0, -300.0, -300.0], np.float32)
    adv = np.array([1.0, 0.0, -1.0, 1.0], np.float32)
    plan = Plan([[4]])
    tiles = _tiles(plan, np.ones(4, np.int32), 0, 0, 0)
    out, _ = _policy_run(tiles, plan, _policy_params(dict(token_advantage=1, reduce=2, loss_scale=1.0)), dev(lp),
                         dev(np.zeros(4, np.float32)), None, None, dev(adv), None, extra=0)
    assert out["grad"].tolist() == [0.0, 0.0, 0.0, 0.0]
    assert out["counts"].tolist() == [[4, 1, 1, 0]]
    # -1.28 + 0 + 0.8 - 0, each term rounded once
    assert abs(float(out["loss"]) - (-1.28 + 0.8)) <= 4 * U * 1.28


def test_policy_gradient_is_the_difference_of_the_loss():
    torch = _torch()
    rng = np.random.default_rng(31)
    plan = Plan([[5, 7], [6]])
    y = plan.labels(rng, 0.3)
    on = plan.counted(y, 1)
    p = _policy_params(dict(kl=3, reduce=1, kl_coef=0.5, entropy_coef=0.1))
    lp = (-rng.random(plan.E)).astype(np.float32)
    old, kref = lp + np.float32(0.1) * rng.standard_normal(plan.E).astype(np.float32), lp - np.float32(0.3)
    H, adv = rng.random(plan.E).astype(np.float32), rng.standard_normal(plan.R).astype(np.float32)
    tiles = _tiles(plan, y, 1, 0, 0)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()

    def loss(lp):
        out, _ = _policy_run(tiles, plan, p, dev(lp), dev(old), dev(kref), dev(H), dev(adv), None, extra=0)
        return out["loss"].double().sum().item(), out["grad"].double().cpu().numpy()
    base, grad = loss(lp)
    for e in np.nonzero(on)[0]:
        up, down = lp.copy(), lp.copy()
        up[e] += 1 / 256
        down[e] -= 1 / 256
        d = (old[e] < lp[e] + np.log1p(0.28) - 1 / 128) and (old[e] > lp[e] - np.log1p(0.28) + 1 / 128)
        if not d:
            continue
        diff = (loss(up)[0] - loss(down)[0]) / (float(up[e]) - float(down[e]))
        # the loss is of size 4, rounded to fp32 with the bound of test_policy_loss, over a step of 2^-7; the
        # third derivative of exp times a step squared / 6 on top
        assert abs(diff - grad[e]) <= 2 * 90 * U * 4 * 128 + 4 * 2.0 ** -16, e


PREFERENCE_OPTIONS = [dict(kind=0), dict(kind=0, label_smoothing=0.2, margin=0.3), dict(kind=1, margin=-0.4),
                      dict(kind=2, beta=0.3), dict(kind=0, normalize=1, beta=2.0), dict(kind=2, normalize=1, ref=False),
                      dict(kind=1, ref=False, beta=0.02)]


def _preference_run(tiles, plan, p, lp, kref, ids, pair, extra=5, extra_rows=3, ws=None, stream=None):
    import paper_2606_19989_amd as odb
    torch = _torch()
    f = lambda *s: torch.full(s, -3.0, device="cuda")
    out = dict(loss=f(1), row_loss=f(plan.R + extra_rows), reward=f(plan.R + extra_rows),
               counts=torch.full((2,), -3, dtype=torch.int64, device="cuda"), grad=f(plan.E + extra))
    if ws is None:
        n = odb.odb_loss_workspace_size(tiles, 0 if ids is None else pair.numel())
        ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    odb.odb_preference_loss(tiles, odb.PreferenceParams(**p), lp, pair, out["loss"], out["row_loss"], out["reward"],
                            out["counts"], ws, ref_logprob=kref, row_ids=ids, grad_logprob=out["grad"], status=status,
                            stream=stream)
    return out, status


def _check_preference(out, want, plan, p, lp, kref, on):
    got = {k: v.double().cpu().numpy() for k, v in out.items()}
    assert np.array_equal(got["counts"], want["counts"])
    R, E = plan.R, plan.E
    assert np.all(got["row_loss"][R:] == -3.0) and np.all(got["reward"][R:] == -3.0) and np.all(got["grad"][E:] == -3.0)
    # everything is formed in 64 bits and rounded once; what 64 bits lose of the sums, times the losses' slopes
    x = np.abs(np.where(on, lp, 0.0).astype(np.float64)) + (0 if kref is None else np.abs(np.where(on, kref, 0.0)))
    lost = 1e-13 * (1 + x.sum()) * (1 + p["beta"]) * (1 + 1 / p["beta"] ** 2) * (1 + np.abs(want["reward"]).max(initial=0))
    near = lambda a, b: np.all(np.abs(a - b) <= 1.01 * U * np.abs(b) + lost)
    assert near(got["row_loss"][:R], want["row_loss"])
    assert near(got["reward"][:R], want["reward"])
    assert near(got["loss"], want["loss"])
    assert near(got["grad"][:E], want["grad"])


@pytest.mark.parametrize("name", list(_plans()))
@pytest.mark.parametrize("by_id", [False, True])
def test_preference_loss(name, by_id):
    torch = _torch()
    plan = _plans()[name]
    for n, o in enumerate(PREFERENCE_OPTIONS):
        log(f"preference loss {name} by_id={by_id} {o}")
        rng = np.random.default_rng(200 + n)
        shift = n % 2
        p = {**dict(kind=0, normalize=0, beta=0.15, margin=0.0, label_smoothing=0.0, loss_scale=0.25),
             **{k: v for k, v in o.items() if k != "ref"}}
        y = plan.labels(rng, 0.4, 0.1)
        on = plan.counted(y, shift)
        lp, kref, _, _ = _inputs(plan, rng, on)
        kref = kref if o.get("ref", True) else None
        num = plan.R + 3 if not by_id else plan.R + 7         # ids without a row here, too
        ids = None
        if by_id:
            ids = rng.permutation(num)[:plan.R].astype(np.int32)
            if plan.R > 4:
                ids[plan.R - 1] = ids[1]                       # an id with two rows: the first counts
        at = rng.permutation(num) if by_id else rng.permutation(plan.R)
        pair = np.zeros(num, np.int32)
        for a, b in zip(at[0::2], at[1::2]):
            if rng.random() < 0.9:
                pair[a], pair[b] = b + 1, -(a + 1)
        want = ref.preference_loss(plan, y, shift, p, lp, kref, ids, pair)
        tiles = _tiles(plan, y, shift)
        idd = None if ids is None else _pad(ids, 3, 10 ** 6)
        out, status = _preference_run(tiles, plan, p, _pad(lp, 5), _pad(kref, 5), idd, torch.from_numpy(pair).cuda())
        assert int(status.item()) == 0
        _check_preference(out, want, plan, p, lp, kref, on)
        again, _ = _preference_run(tiles, plan, p, _pad(lp, 5), _pad(kref, 5), idd, torch.from_numpy(pair).cuda())
        for k, v in out.items():
            assert torch.equal(v, again[k]), k


def test_preference_far_margins_stay_finite():
    torch = _torch()
    plan = Plan([[2, 2, 2, 2]])
    y = np.ones(plan.E, np.int32)
    lp = np.array([0, 0, -5000, -5000, -5000, -5000, 0, 0], np.float32)
    pair = np.array([2, -1, 4, -3], np.int32)
    for kind in (0, 1):
        p = dict(kind=kind, normalize=0, beta=1.0, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
        want = ref.preference_loss(plan, y, 0, p, lp, None, None, pair)
        tiles = _tiles(plan, y, 0, 0, 0)
        out, _ = _preference_run(tiles, plan, p, torch.from_numpy(lp).cuda(), None, None, torch.from_numpy(pair).cuda(),
                                 0, 0)
        _check_preference(out, want, plan, p, lp, None, y == 1)
        assert out["row_loss"].tolist() == [0.0, 0.0, 10000.0 + kind, 0.0]


def test_labels_without_probability_in_a_pair():
    """Log ratios of -inf and +inf: the loss of the pair's right order is 0, the other's infinite."""
    torch = _torch()
    inf = math.inf
    plan = Plan([[2, 2, 2, 2]])
    lp = np.array([-1, -1, -inf, -1, -1, -inf, -1, -1], np.float32)      # row 1 and row 2
    pair = np.array([2, -1, 4, -3], np.int32)                             # 0 over 1, 2 over 3
    tiles = _tiles(plan, np.ones(plan.E, np.int32), 0, 0, 0)
    dev = lambda x: torch.from_numpy(x).cuda()
    for kind, smoothing, losses, slopes in ((0, 0.0, (0.0, inf), (0.0, -0.5)), (0, 1.0, (inf, 0.0), (0.5, 0.0)),
                                            (0, 0.25, (inf, inf), (0.125, -0.375)), (1, 0.0, (0.0, inf), (0.0, -0.5))):
        p = dict(kind=kind, normalize=0, beta=0.5, margin=0.0, label_smoothing=smoothing, loss_scale=1.0)
        out, status = _preference_run(tiles, plan, p, dev(lp), None, None, dev(pair), 0, 0)
        assert int(status.item()) == 0
        assert out["row_loss"].tolist() == [losses[0], 0.0, losses[1], 0.0]
        assert out["reward"].tolist() == [-1.0, -inf, -inf, -1.0] and out["counts"].tolist() == [2, 1]
        a, b = slopes
        assert out["grad"].tolist() == [a, a, -a, -a, b, b, -b, -b]


def test_watched_kl_term_may_overflow():
    """With a coefficient of 0 the KL term is only reported: neither the loss nor the gradient takes part in it."""
    torch = _torch()
    dev = lambda x: torch.from_numpy(x).cuda()
    for groups in ([[4]], [[4], [5000]]):         # one launch, and the passes
        plan = Plan(groups)
        lp, kref = np.full(plan.E, -1.0, np.float32), np.full(plan.E, -1.0, np.float32)
        kref[1] = 120.0                            # exp(121) passes fp32
        tiles = _tiles(plan, np.ones(plan.E, np.int32), 0, 0, 0)
        for reduce in range(3):
            out, _ = _policy_run(tiles, plan, _policy_params(dict(kl=3, reduce=reduce, kl_coef=0.0, loss_scale=1.0)),
                                 dev(lp), dev(lp), dev(kref), None, dev(np.full(plan.R, 2.0, np.float32)), None, extra=0)
            n = 1 if reduce == 2 else 4
            assert out["grad"][:4].tolist() == [-2.0 / n] * 4
            assert out["loss"].tolist() == [-2.0 * (plan.tile_off[k + 1] - plan.tile_off[k] if reduce == 2 else 1)
                                            for k in range(plan.K)]
            assert out["means"][0, 1].item() == math.inf
            H = np.ones(plan.E, np.float32)
            H[2] = np.inf
            out, _ = _policy_run(tiles, plan, _policy_params(dict(kl=0, reduce=reduce, loss_scale=1.0)), dev(lp), dev(lp),
                                 None, dev(H), dev(np.full(plan.R, 2.0, np.float32)), None, extra=0)
            assert bool(torch.isfinite(out["loss"]).all()) and out["means"][0, 2].item() == math.inf
            assert out["grad"][:4].tolist() == [-2.0 / n] * 4


def test_policy_terms_that_nearly_cancel():
    """Ratios of 1 and advantages of few bits, so that every term is exact: what is left of terms a million
    times larger is rounded once."""
    torch = _torch()
    dev = lambda x: torch.from_numpy(x).cuda()
    rng = np.random.default_rng(61)
    for lens in ([3, 5, 7, 11], [int(v) for v in rng.integers(1, 90, 40)], [int(v) for v in rng.integers(100, 900, 40)]):
        plan = Plan([lens])
        y = plan.labels(rng)
        on = plan.counted(y, 0)
        lp = -rng.random(plan.E).astype(np.float32)
        adv = (rng.integers(-4096, 4097, plan.R) / 1024.0).astype(np.float32)
        count = np.array([on[plan.row_of == r].sum() for r in range(plan.R)])
        for reduce, weight in ((0, count / count.sum()), (1, np.full(plan.R, 1 / plan.R)), (2, count.astype(np.float64))):
            # the last row's advantage takes back the others', up to its own step
            adv[-1] = np.float32(np.round(-(adv[:-1].astype(np.float64) * weight[:-1]).sum() / weight[-1] * 1024) / 1024)
            tiles = _tiles(plan, y, 0, 0, 0)
            out, _ = _policy_run(tiles, plan, _policy_params(dict(kl=0, reduce=reduce, loss_scale=1.0, clip_low=0.5,
                                                                  clip_high=0.5)), dev(lp), dev(lp), None, None,
                                 dev(adv), None, extra=0)
            want = -(adv.astype(np.float64) * weight).sum()
            lost = 1e-15 * (np.abs(adv) * weight).sum() * plan.E
            assert abs(float(out["loss"]) - want) <= U * abs(want) + lost, (plan.E, reduce)


def test_calls_without_gradients():
    """Values alone: the same bits as beside gradients, in every path by the run's size."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    for groups in ([[5, 9, 3]], [[700] * 9, [650] * 8], [[30] * 400, [7] * 300]):
        plan = Plan(groups)
        log(f"without gradients: {plan.E} elements")
        rng = np.random.default_rng(5)
        y = plan.labels(rng, 0.3)
        on = plan.counted(y, 1)
        lp, old, kref, H = (torch.from_numpy(np.where(on, v, 0).astype(np.float32)).cuda() for v in
                            _inputs(plan, rng, on))
        adv = torch.from_numpy(rng.standard_normal(plan.R).astype(np.float32)).cuda()
        tiles = _tiles(plan, y, 1, 0, 0)
        ws = torch.empty(odb.odb_loss_workspace_size(tiles, plan.R), dtype=torch.uint8, device="cuda")
        for reduce in range(3):
            p = _policy_params(dict(kl=3, reduce=reduce, entropy_coef=0.1))
            want, _ = _policy_run(tiles, plan, p, lp, old, kref, H, adv, None, extra=0)
            for with_grad in (False, True):           # entropies without their gradient
                got = [torch.empty_like(want[k]) for k in ("loss", "means", "counts", "grad")]
                odb.odb_policy_loss(tiles, odb.PolicyParams(**p), lp, adv, *got[:3], ws, old_logprob=old, ref_logprob=kref,
                                    entropy=H, grad_logprob=got[3] if with_grad else None)
                for k, v in zip(("loss", "means", "counts", "grad")[:4 if with_grad else 3], got):
                    assert torch.equal(v, want[k]), (reduce, k)
        at = rng.permutation(plan.R)[:plan.R // 2 * 2]
        pair = np.zeros(plan.R, np.int32)
        pair[at[0::2]], pair[at[1::2]] = at[1::2] + 1, -(at[0::2] + 1)
        pair = torch.from_numpy(pair).cuda()
        for ids in (None, torch.arange(plan.R, dtype=torch.int32, device="cuda")):
            p = dict(kind=0, normalize=0, beta=0.2, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
            want, _ = _preference_run(tiles, plan, p, lp, kref, ids, pair, 0, 0)
            got = [torch.empty_like(want[k]) for k in ("loss", "row_loss", "reward", "counts")]
            odb.odb_preference_loss(tiles, odb.PreferenceParams(**p), lp, pair, *got, ws, ref_logprob=kref, row_ids=ids)
            for k, v in zip(("loss", "row_loss", "reward", "counts"), got):
                assert torch.equal(v, want[k]), k


@pytest.mark.parametrize("elems", [0, 3000, 40_000])
def test_many_idle_slots(elems):
    """300,000 slots, nearly all of them idle: before, between and behind those with rows."""
    torch = _torch()
    log(f"idle slots, {elems} elements")
    rng = np.random.default_rng(elems)
    lens = []
    while sum(lens) < elems:
        lens.append(int(rng.integers(1, 120)))
    groups = [[] for _ in range(300_000)]
    for l, k in zip(lens, sorted(rng.choice(np.arange(50, 299_000), len(lens), replace=False))):
        groups[k] = [l, l]
    plan = Plan(groups)
    y = plan.labels(rng, 0.3)
    on = plan.counted(y, 0)
    lp, old, kref, _ = (np.where(on, v, 0).astype(np.float32) for v in _inputs(plan, rng, on))
    adv = rng.standard_normal(plan.R).astype(np.float32)
    tiles = _tiles(plan, y, 0, 0, 0)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    for reduce in range(3):
        p = _policy_params(dict(kl=3, reduce=reduce))
        want = ref.policy_loss(plan, y, 0, p, lp, old, kref, None, adv, None)
        out, status = _policy_run(tiles, plan, p, dev(lp), dev(old), dev(kref), None, dev(adv), None, extra=0)
        assert int(status.item()) == 0
        assert np.array_equal(out["counts"].cpu().numpy(), want["counts"])
        # the bound of test_policy_loss for ratios of at most exp(10)
        C = 100 * U
        mag = p["loss_scale"] * (want["mags"][:, 0] + p["kl_coef"] * want["mags"][:, 1])
        assert np.all(np.abs(out["loss"].double().cpu().numpy() - want["loss"]) <= C * mag + 2 * U * np.abs(want["loss"]))
        assert np.all(np.abs(out["grad"].double().cpu().numpy() - want["grad"]) <= 2 * C * want["grad_mag"])
    pair = np.zeros(plan.R, np.int32)
    pair[0::2], pair[1::2] = np.arange(1, plan.R, 2) + 1, -(np.arange(0, plan.R, 2) + 1)
    p = dict(kind=0, normalize=0, beta=0.2, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
    for ids in (None, np.arange(plan.R, dtype=np.int32)):
        want = ref.preference_loss(plan, y, 0, p, lp, kref, ids, pair)
        out, status = _preference_run(tiles, plan, p, dev(lp), dev(kref), None if ids is None else dev(ids), dev(pair), 0, 0)
        assert int(status.item()) == 0
        _check_preference(out, want, plan, p, lp, kref, on)


def test_bad_pairs_are_reported_and_do_not_count():
    torch = _torch()
    plan = Plan([[3, 4], [5, 6]])
    y = np.ones(plan.E, np.int32)
    lp = np.full(plan.E, -1.0, np.float32)
    p = dict(kind=0, normalize=0, beta=0.1, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
    tiles = _tiles(plan, y, 0, 0, 0)
    dev = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()
    lpd = torch.from_numpy(lp).cuda()
    for pair, pairs in (([2, -1, 0, 0], 1), ([2, 1, 4, -3], 1), ([2, 0, 0, 0], 0), ([1, 0, 0, 0], 0),
                        ([5, 0, 0, 0], 0), ([-5, 0, 0, 0], 0), ([2 ** 31 - 1, -2 ** 31, 4, -3], 1), ([2, -3, -2, 0], 0)):
        for ids in (None, dev([0, 1, 2, 3])):
            out, status = _preference_run(tiles, plan, p, lpd, None, ids, dev(pair), 0, 0)
            assert (int(status.item()) != 0) == (pair != [2, -1, 0, 0]), pair
            assert out["counts"].tolist()[0] == pairs, pair
    for ids in ([0, 1, 2, 4], [0, 1, -1, 3], [2 ** 31 - 1, 1, 0, -2 ** 31]):     # ids out of range
        out, status = _preference_run(tiles, plan, p, lpd, None, dev(ids), dev([2, -1, 0, 0]), 0, 0)
        assert int(status.item()) != 0
        assert out["counts"].tolist()[0] == 1


def test_contradicting_tiles_are_reported():
    """Bounds hold on the host test's arrays; here the status word and the sound slots."""
    torch = _torch()
    plan = Plan([[4, 6], [9], [3, 3, 3]])
    rng = np.random.default_rng(2)
    y = plan.labels(rng)
    on = plan.counted(y, 1)
    lp, old, kref, H = (np.where(on, v, 0).astype(np.float32) for v in _inputs(plan, rng, on))
    adv = rng.standard_normal(plan.R).astype(np.float32)
    p = _policy_params(dict(kl=3, reduce=1))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    want = ref.policy_loss(plan, y, 1, p, lp, old, kref, None, adv, None)
    pp = dict(kind=0, normalize=0, beta=0.1, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
    for field, at, value, sound in (("rows", 1, 2, [0, 2]), ("maxlen", 1, 8, [0, 2]), ("rows", 2, -3, [0, 1]),
                                    ("tile_off", 3, 1000, [0, 1]), ("row_off", 3, 7, [0, 1]), ("maxlen", 0, 0, [1, 2]),
                                    ("row_off", 1, -5, [2]), ("tile_off", 2, -1, [0])):
        bad = Plan([[4, 6], [9], [3, 3, 3]])
        getattr(bad, field)[at] = value
        tiles = _tiles(bad, y, 1, 0, 0)
        out, status = _policy_run(tiles, plan, p, dev(lp), dev(old), dev(kref), None, dev(adv), None, extra=0)
        assert int(status.item()) != 0, (field, at)
        for k in sound:
            assert abs(float(out["loss"][k]) - want["loss"][k]) <= 100 * U * (1 + abs(want["loss"][k])), (field, at, k)
            a, b = plan.tile_off[k], plan.tile_off[k + 1]
            assert np.allclose(out["grad"].cpu().numpy()[a:b], want["grad"][a:b], rtol=1e-4, atol=1e-6)
        out, status = _preference_run(tiles, plan, pp, dev(lp), None, None, dev(np.zeros(plan.R, np.int32)), 0, 0)
        assert int(status.item()) != 0, (field, at)


@pytest.mark.parametrize("elems", [60_000, 3_000_000, 6_000_000, 9_000_000, 34_000_000])
def test_large_runs(elems):
    """Runs of many tiles whose rows divide, or nearly divide, every step of the kernels, and whose
    tiles start at any element; each size takes another length of chunk."""
    torch = _torch()
    rng = np.random.default_rng(elems)
    lens = [1, 2, 3, 4, 5, 7, 8, 16, 31, 32, 33, 64, 65, 100, 128, 255, 256, 257, 341, 480, 511, 512, 513, 1000, 1023,
            1024, 1025, 2048, 4096, 4097, 5000, 8192]
    groups, total, k = [], 0, 0
    while total < elems:
        l = lens[k % len(lens)] if k < 4 * len(lens) else int(rng.integers(1, 1500))
        n = max(1, int(rng.integers(1000, min(60_000, elems // 20)) // l))
        if l == 1:
            n = min(n, 3000)
        groups.append([max(1, l - int(v)) for v in rng.integers(0, 1 + l // 9, n - 1)] + [l])
        total += n * l
        k += 1
        if k % 7 == 0:
            groups.append([])
    plan = Plan(groups, base=(11, 1 << 34))
    log(f"large run: {plan.K} tiles, {plan.R} rows, {plan.E} elements")
    y_host = plan.labels(rng, 0.3, 0.05)
    tiles = _tiles(plan, y_host, 1, 0, 0)
    y = tiles.labels
    maps = ref.Maps(plan, "cuda")
    gen = torch.Generator("cuda").manual_seed(elems)
    r = lambda n, sd: torch.randn(n, generator=gen, device="cuda") * sd
    lp = -r(plan.E, 2).abs()
    old, kref, adv = lp + r(plan.E, 0.2), lp + r(plan.E, 0.4), r(plan.R, 1)
    for reduce in range(3):
        p = _policy_params(dict(kl=3, reduce=reduce))
        out, status = _policy_run(tiles, plan, p, lp, old, kref, None, adv, None, extra=0)
        assert int(status.item()) == 0
        want = ref.policy_loss_torch(maps, y, 1, p, lp, old, kref, adv)
        assert torch.equal(out["counts"], want["counts"])
        C = (80 + 2 * 2) * U        # no ratio is further off than exp(2): 10 standard deviations
        mag = p["loss_scale"] * (want["mags"][:, 0] + p["kl_coef"] * want["mags"][:, 1])
        assert torch.all((out["loss"].double() - want["loss"]).abs() <= C * mag + 2 * U * want["loss"].abs())
        assert torch.all((out["means"].double() - want["means"]).abs() <= C * want["mags"] + 1e-12)
        assert torch.all((out["grad"].double() - want["grad"]).abs() <= 2 * C * want["grad_mag"])
        again, _ = _policy_run(tiles, plan, p, lp, old, kref, None, adv, None, extra=0)
        for key, v in out.items():
            assert v is None or torch.equal(v, again[key]), key
    ids = torch.randperm(plan.R, generator=gen, device="cuda").int()
    at = torch.randperm(plan.R, generator=gen, device="cuda")
    pair = torch.zeros(plan.R, dtype=torch.int32, device="cuda")
    a, b = at[0:plan.R // 2 * 2:2], at[1:plan.R // 2 * 2:2]
    pair[a], pair[b] = (b + 1).int(), -(a + 1).int()
    p = dict(kind=0, normalize=0, beta=0.05, margin=0.0, label_smoothing=0.0, loss_scale=0.125)
    out, status = _preference_run(tiles, plan, p, lp, kref, ids, pair, 0, 0)
    assert int(status.item()) == 0
    want = ref.preference_loss_torch(maps, y, 1, p, lp, kref, ids, pair)
    # 64-bit sums of at most 8,192 terms of size 10, rounded once; the total adds 2^20 of them
    near = lambda x, w: torch.all((x.double() - w).abs() <= 1.01 * U * w.abs() + 1e-9)
    assert torch.equal(out["counts"], want["counts"])
    assert near(out["row_loss"], want["row_loss"]) and near(out["reward"], want["reward"])
    assert near(out["grad"], want["grad"]) and near(out["loss"], want["loss"].reshape(1))


LONG_ROWS = {"two": [[65_536, 131_072]], "beside_short": [[3, 40_000], [70_001, 5, 70_000, 69_999], [20], [30_000]],
             "many": [[40_000 + 7 * i for i in range(40)], [5] * 30, [9_000] * 20], "one": [[400_000]]}


@pytest.mark.parametrize("name", list(LONG_ROWS))
def test_long_rows(name):
    """Rows over many chunks, prompts that fill whole chunks, and a row in which nothing counts."""
    torch = _torch()
    plan = Plan(LONG_ROWS[name], base=(5, 77))
    log(f"long rows {name}: {plan.R} rows, {plan.E} elements")
    rng = np.random.default_rng(83)
    y_host = plan.labels(rng, 0.9)
    y_host[plan.row_of == plan.R - 1] = IGNORE if plan.R > 1 else 1
    tiles = _tiles(plan, y_host, 0, 0, 0)
    y = tiles.labels
    maps = ref.Maps(plan, "cuda")
    gen = torch.Generator("cuda").manual_seed(83)
    r = lambda n, sd: torch.randn(n, generator=gen, device="cuda") * sd
    lp = -r(plan.E, 2).abs()
    old, kref, adv = lp + r(plan.E, 0.2), lp + r(plan.E, 0.4), r(plan.R, 1)
    for reduce in range(3):
        p = _policy_params(dict(kl=3, reduce=reduce))
        out, status = _policy_run(tiles, plan, p, lp, old, kref, None, adv, None, extra=0)
        assert int(status.item()) == 0
        want = ref.policy_loss_torch(maps, y, 0, p, lp, old, kref, adv)
        assert torch.equal(out["counts"], want["counts"])
        C = (80 + 2 * 2) * U        # as in test_large_runs
        mag = p["loss_scale"] * (want["mags"][:, 0] + p["kl_coef"] * want["mags"][:, 1])
        assert torch.all((out["loss"].double() - want["loss"]).abs() <= C * mag + 2 * U * want["loss"].abs())
        assert torch.all((out["grad"].double() - want["grad"]).abs() <= 2 * C * want["grad_mag"])
    ids = torch.randperm(plan.R, generator=gen, device="cuda").int()
    pair = torch.zeros(plan.R, dtype=torch.int32, device="cuda")
    at = torch.randperm(plan.R, generator=gen, device="cuda")
    a, b = at[0:plan.R // 2 * 2:2], at[1:plan.R // 2 * 2:2]
    pair[a], pair[b] = (b + 1).int(), -(a + 1).int()
    for normalize, beta in ((0, 1e-4), (1, 2.0)):
        p = dict(kind=0, normalize=normalize, beta=beta, margin=0.0, label_smoothing=0.0, loss_scale=0.125)
        out, status = _preference_run(tiles, plan, p, lp, kref, ids, pair, 0, 0)
        assert int(status.item()) == 0
        want = ref.preference_loss_torch(maps, y, 0, p, lp, kref, ids, pair)
        # 64-bit sums of at most 400,000 terms of size 10, times a factor of at most 2, rounded once
        near = lambda x, w: torch.all((x.double() - w).abs() <= 1.01 * U * w.abs() + 1e-9)
        assert torch.equal(out["counts"], want["counts"])
        assert near(out["row_loss"], want["row_loss"]) and near(out["reward"], want["reward"])
        assert near(out["grad"], want["grad"]) and near(out["loss"], want["loss"].reshape(1))
        again, _ = _preference_run(tiles, plan, p, lp, kref, ids, pair, 0, 0)
        for key, v in out.items():
            assert torch.equal(v, again[key]), key


def test_tiles_past_32_bits():
    """More than 2^31 elements in one slot of two rows: positions, the mean and the last elements."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    L = (1 << 30) + 5
    E = 2 * L
    log(f"tiles past 32 bits: 2 x {L}")
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    y = torch.ones(E, **i32)
    y[L - 3:L] = IGNORE
    tiles = odb.Tiles(torch.tensor([2], **i32), torch.tensor([L], **i32), torch.tensor([0, 2], **i64),
                      torch.tensor([0, E], **i64), y, 2)
    ws = torch.empty(odb.odb_loss_workspace_size(tiles), dtype=torch.uint8, device="cuda")
    lp = torch.full((E,), -0.5, device="cuda")
    grad = torch.full((E,), 7.0, device="cuda")
    adv = torch.tensor([1.0, -2.0], device="cuda")
    loss, means, counts = (torch.empty(1, device="cuda"), torch.empty(1, 4, device="cuda"),
                           torch.empty(1, 4, **i64))
    status = torch.zeros(1, **i32)
    for reduce, n in ((0, None), (1, None)):
        odb.odb_policy_loss(tiles, odb.PolicyParams(reduce=reduce, loss_scale=1e9), lp, adv, loss, means, counts, ws,
                            grad_logprob=grad, status=status)
        assert int(status.item()) == 0
        a, b = L - 1 - 3, L - 1                     # counted tokens of the rows
        assert counts.tolist() == [[a + b, 0, 0, 0]]
        w0, w1 = (1 / (a + b), 1 / (a + b)) if reduce == 0 else (1 / (2 * a), 1 / (2 * b))
        want = -1e9 * (w0 * a - 2 * w1 * b)
        assert abs(float(loss) - want) <= 4 * U * 1e9 * 3
        for at, g in ((0, 0.0), (1, -1e9 * w0), (L - 4, -1e9 * w0), (L - 3, 0.0), (L - 1, 0.0), (L, 0.0),
                      (L + 1, 2e9 * w1), (E - 1, 2e9 * w1)):
            assert abs(float(grad[at]) - g) <= 4 * U * abs(g), at
        assert int((grad == 0).sum()) == 5
    pair = torch.tensor([2, -1], **i32)
    row = [torch.empty(2, device="cuda") for _ in range(2)]
    pc = torch.empty(2, **i64)
    odb.odb_preference_loss(tiles, odb.PreferenceParams(beta=1e-9), lp, pair, loss, row[0], row[1], pc, ws,
                            grad_logprob=grad, status=status)
    assert int(status.item()) == 0 and pc.tolist() == [1, 1]
    assert abs(float(row[1][0]) + 0.5e-9 * a) <= 2 * U * 0.6 and abs(float(row[1][1]) + 0.5e-9 * b) <= 2 * U * 0.6
    assert float(grad[L + 1]) > 0 > float(grad[1]) and float(grad[E - 1]) == float(grad[L + 1])


# ------------------------------------------------------------------------- streams and graphs
def _step(odb, torch, s):
    """What a trainer does with one tile, all outputs kept."""
    odb.odb_token_logprobs(s["z"], s["y"], s["lp"], stats=s["st"], entropy=s["H"], stream=s.get("stream"))
    odb.odb_policy_loss(s["tiles"], s["params"], s["lp"], s["adv"], s["loss"], s["means"], s["counts"], s["ws"],
                        old_logprob=s["old"], ref_logprob=s["ref"], entropy=s["H"], grad_logprob=s["g"],
                        grad_entropy=s["gH"], stream=s.get("stream"))
    odb.odb_token_logprobs_backward(s["z"], s["y"], s["st"], s["g"], s["dz"], entropy=s["H"], grad_entropy=s["gH"],
                                    stream=s.get("stream"))
    odb.odb_preference_loss(s["tiles"], s["pref"], s["lp"], s["pair"], s["ploss"], s["rl"], s["rr"], s["pc"], s["ws"],
                            ref_logprob=s["ref"], row_ids=s["ids"], grad_logprob=s["pg"], stream=s.get("stream"))


def _step_state(odb, torch, rows, cols, V, seed, reduce=1):
    gen = torch.Generator("cuda").manual_seed(seed)
    f = lambda *s: torch.empty(*s, device="cuda")
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    y = torch.randint(0, V, (rows, cols), generator=gen, **i32)
    y[:, :2] = IGNORE
    tiles = odb.Tiles(torch.tensor([rows], **i32), torch.tensor([cols], **i32), torch.tensor([0, rows], **i64),
                      torch.tensor([0, rows * cols], **i64), y, rows)
    pair = torch.zeros(rows, **i32)
    pair[0::2] = torch.arange(1, rows, 2, **i32) + 1
    pair[1::2] = -(torch.arange(0, rows, 2, **i32) + 1)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return dict(z=r(rows, cols, V).bfloat16(), y=y, lp=f(rows, cols), st=f(rows, cols, 2), H=f(rows, cols), tiles=tiles,
                params=odb.PolicyParams(kl=3, reduce=reduce, kl_coef=0.1, entropy_coef=0.01),
                pref=odb.PreferenceParams(), adv=r(rows), old=r(rows, cols) * 0.2 - 5, ref=r(rows, cols) * 0.2 - 5,
                loss=f(1), means=f(4), counts=torch.empty(4, **i64), g=f(rows, cols), gH=f(rows, cols),
                dz=torch.empty(rows, cols, V, dtype=torch.bfloat16, device="cuda"), pair=pair,
                ids=torch.arange(rows, **i32), ploss=f(1), rl=f(rows), rr=f(rows), pc=torch.empty(2, **i64),
                pg=f(rows, cols), ws=torch.empty(odb.odb_loss_workspace_size(tiles, rows), dtype=torch.uint8,
                                                 device="cuda"))


OUTPUTS = ("lp", "st", "H", "loss", "means", "counts", "g", "gH", "dz", "ploss", "rl", "rr", "pc", "pg")


@pytest.mark.parametrize("shape", [(4, 9, 50), (6, 700, 3000)], ids=str)
def test_step_in_a_graph_and_on_streams(shape):
    import paper_2606_19989_amd as odb
    torch = _torch()
    log(f"step in a graph {shape}")
    s = _step_state(odb, torch, *shape, seed=1)
    other = _step_state(odb, torch, *shape, seed=2, reduce=0)
    eager = {}
    for seed in (1, 3, 4):
        v = _step_state(odb, torch, *shape, seed=seed)
        _step(odb, torch, v)
        eager[seed] = {k: v[k].clone() for k in OUTPUTS} | {k: v[k] for k in ("z", "y", "adv", "old", "ref")}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        _step(odb, torch, s)          # loads the kernels
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        _step(odb, torch, s)
    for seed in (3, 1, 4, 1):
        for k in ("z", "y", "adv", "old", "ref"):
            s[k].copy_(eager[seed][k])
        for k in OUTPUTS:
            s[k].zero_()
        torch.cuda.synchronize()
        _step(odb, torch, other)      # eager work with a workspace of its own between the replays
        graph.replay()
        torch.cuda.synchronize()
        for k in OUTPUTS:
            assert torch.equal(s[k], eager[seed][k]), (seed, k)
    # two streams at once, each with its own workspace
    a, b = _step_state(odb, torch, *shape, seed=3), _step_state(odb, torch, *shape, seed=4)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        _step(odb, torch, dict(a, stream=sa))
        _step(odb, torch, dict(b, stream=sb))
    torch.cuda.synchronize()
    for k in OUTPUTS:
        assert torch.equal(a[k], eager[3][k]) and torch.equal(b[k], eager[4][k]), k


def test_binding_checks_types_and_sizes():
    import paper_2606_19989_amd as odb
    torch = _torch()
    s = _step_state(odb, torch, 4, 9, 50, seed=1)
    for k, bad in (("lp", s["lp"].double()), ("lp", s["lp"][:2]), ("st", s["lp"]), ("y", s["y"].long()),
                   ("H", s["H"].half())):
        with pytest.raises(ValueError):
            odb.odb_token_logprobs(s["z"], bad if k == "y" else s["y"], bad if k == "lp" else s["lp"],
                                   stats=bad if k == "st" else s["st"], entropy=bad if k == "H" else s["H"])
    with pytest.raises(ValueError):
        odb.odb_token_logprobs(s["z"], s["y"].t(), s["lp"])       # labels must be contiguous
    with pytest.raises(ValueError):
        odb.odb_token_logprobs_backward(s["z"], s["y"], s["st"], s["g"], s["dz"][:, :, :40])
    with pytest.raises(ValueError):
        odb.odb_token_logprobs_backward(s["z"], s["y"], s["st"], s["g"], s["dz"].float())
    for wide in (torch.zeros(4, 10, dtype=torch.int32, device="cuda"), torch.zeros(5, 9, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError, match="labels"):           # another tile's
            odb.odb_token_logprobs(s["z"], wide, s["lp"])
    odb.odb_token_logprobs(s["z"], torch.zeros(40, dtype=torch.int32, device="cuda"), s["lp"])    # flat and longer

    class Elsewhere:
        cuda_stream, device_index = 0, 1
    for call in (lambda: odb.odb_token_logprobs(s["z"], s["y"], s["lp"], stream=Elsewhere),
                 lambda: odb.odb_policy_loss(s["tiles"], s["params"], s["lp"], s["adv"], s["loss"], s["means"],
                                             s["counts"], s["ws"], entropy=s["H"], ref_logprob=s["ref"],
                                             stream=Elsewhere)):
        with pytest.raises(ValueError, match="stream"):
            call()


# ------------------------------------------------------------------------- the whole chain
def _chain(pipe, w_ranks, ids, V, seed):
    """Collate, then per tile: a linear model's logits, their log-probabilities; a policy loss with
    the plan's loss weights and a preference loss over the whole plan; the gradients back to every
    tile's logits.  Everything again in 64 bits on the CPU by torch's differentiation."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    labels = pipe.collate()[1]
    K, P = pipe.num_slots, int(pipe.info["padded_elems"])
    rows, maxlen = pipe.slot_rows[:K].tolist(), pipe.slot_maxlen[:K].tolist()
    off = pipe.slot_tile_off[:K + 1].tolist()
    gen = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    labels.copy_(torch.where(labels != IGNORE, labels % V, labels))       # the tiny model's vocabulary
    z = rnd(P, V) * 2
    lp, st, H = torch.empty(P, device="cuda"), torch.empty(P, 2, device="cuda"), torch.empty(P, device="cuda")
    tile = lambda x, k: x[off[k]:off[k + 1]].view(rows[k], maxlen[k], *x.shape[1:])
    for k in range(K):
        if rows[k]:
            odb.odb_token_logprobs(tile(z, k), tile(labels, k), tile(lp, k), stats=tile(st, k), entropy=tile(H, k))
    R = pipe.tiles().num_rows
    adv, old, kref = rnd(R), lp + 0.3 * rnd(P), lp + 0.5 * rnd(P)
    perm = torch.randperm(ids, generator=gen, device="cuda")
    pair = torch.zeros(ids, dtype=torch.int32, device="cuda")
    a, b = perm[0:ids // 2 * 2:2], perm[1:ids // 2 * 2:2]
    pair[a], pair[b] = (b + 1).int(), -(a + 1).int()
    tiles = pipe.tiles(labels)
    weight = pipe.loss_weights(odb.ODB_WEIGHT_TOKEN_EXACT)[0]
    p = odb.PolicyParams(kl=odb.ODB_KL_EXP, reduce=odb.ODB_REDUCE_TOKEN_MEAN, kl_coef=0.1, entropy_coef=0.02,
                         loss_scale=float(w_ranks))
    loss, means, counts, g, gH = pipe.policy_loss(tiles, lp, adv, p, old, kref, H, weight)
    q = odb.PreferenceParams(beta=0.05, loss_scale=0.1)
    ploss, row_loss, reward, pcounts, pg = pipe.preference_loss(tiles, lp, pair, q, kref)
    total = g + pg
    dz = torch.empty_like(z)
    for k in range(K):
        if rows[k]:
            odb.odb_token_logprobs_backward(tile(z, k), tile(labels, k), tile(st, k), tile(total, k), tile(dz, k),
                                            entropy=tile(H, k), grad_entropy=tile(gH, k))
    pipe.check_losses()

    # 64 bits, from the logits to both losses
    zc = z.double().cpu().requires_grad_()
    yc = labels.cpu().long()
    row_max = torch.repeat_interleave(torch.tensor(maxlen), torch.tensor(rows))
    start = torch.cumsum(row_max, 0) - row_max
    row = torch.repeat_interleave(torch.arange(R), row_max)
    col = torch.arange(P) - start[row]
    slot = torch.repeat_interleave(torch.arange(K), torch.tensor(rows))[row]
    on = torch.nonzero((yc != IGNORE) & (col >= 1))[:, 0]
    lq = torch.log_softmax(zc[on - 1], -1)
    c_lp = lq.gather(1, yc[on, None])[:, 0]
    c_H = -(lq.exp() * lq).sum(-1)
    A, d = adv.cpu().double()[row[on]], c_lp - old.cpu().double()[on]
    r = d.exp()
    pol = -torch.minimum(r * A, r.clamp(0.8, 1.2) * A)
    x = c_lp - kref.cpu().double()[on]
    n = torch.bincount(slot[on], minlength=K).double()
    per = weight.cpu()[slot[on]] * w_ranks / n[slot[on]]
    val = per * (pol + 0.1 * (torch.exp(-x) + x - 1) - 0.02 * c_H)
    c_loss = torch.zeros(K, dtype=torch.float64).index_add(0, slot[on], val)
    S = torch.zeros(R, dtype=torch.float64).index_add(0, row[on], x)
    emit = pipe.emit_order[:R].cpu().long()
    first = {}
    for i, v in enumerate(emit.tolist()):
        first.setdefault(v, i)
    pc = [(first[int(v)], first[int(pair[v]) - 1]) for v in torch.nonzero(pair > 0)[:, 0].tolist()
          if v in first and int(pair[v]) - 1 in first]
    h = 0.05 * (S[[i for i, _ in pc]] - S[[j for _, j in pc]])
    c_ploss = -0.1 * torch.nn.functional.logsigmoid(h).sum()
    (c_loss.sum() + c_ploss).backward()
    c_ploss, x = c_ploss.detach(), x.detach()
    assert pcounts.tolist()[0] == len(pc) and counts[:, 0].tolist() == n.long().tolist()
    # a log-probability is off by (V / 64 + 60) U at most, the terms built on it by as much relatively; sums of
    # at most P of them, weighted
    e = (V / 64 + 60 + 40) * U
    mag = torch.zeros(K, dtype=torch.float64).index_add(0, slot[on], per * (pol.abs() + r * A.abs() + 0.1 * (
        torch.exp(-x) + x.abs()) + 0.02 * (c_H + 1))).detach()
    assert torch.all((loss.cpu().double() - c_loss.detach()).abs() <= 4 * e * mag + 1e-12)
    assert abs(float(ploss) - float(c_ploss)) <= 2 * e * (0.1 * len(pc) + 0.1 * 0.05 * float(x.abs().sum()))
    want = zc.grad
    # tokens whose ratio lies within the error of a clip may fall on either side
    edge = torch.zeros(P, dtype=torch.bool)
    edge[on - 1] = ((d - math.log(1.2)).abs() < 20 * e) | ((d - math.log(0.8)).abs() < 20 * e)
    err = (dz.cpu().double() - want).abs()
    # the gradient's factor on the logits is at most that of the log-probability, p and 1 - p are below 1
    top = torch.zeros(P, dtype=torch.float64)
    top[on - 1] = (per * (r * A.abs() + 0.1 * (torch.exp(-x) + x.abs() + 1) + 0.1 * (c_H + 1))).detach() + 0.005
    assert torch.all(err[~edge] <= 10 * e * top[~edge, None])
    assert torch.any(dz != 0)
    return tiles, lp, adv, p, old, kref, H, weight, loss, g


@pytest.mark.parametrize("mode", ["join", "nonjoin"])
def test_chain_behind_a_window(mode):
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(71)
    w = synth.window_from_ranks("loss_chain", [rng.integers(2, 90, 60), rng.integers(2, 90, 41),
                                               rng.integers(2, 40, 7)], 400)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")
    pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget, mode=mode,
                        quota=80)
    pipe.form()
    pipe.align()
    log(f"chain behind a window: {mode}, {pipe.num_slots} slots")
    tiles, lp, adv, p, old, kref, H, weight, loss, g = _chain(pipe, w.W, w.n, 89, 5)
    loss, g = loss.clone(), g.clone()
    # tile by tile, as ranks call it: the same numbers as the whole plan's
    for k in (0, 1, pipe.num_slots - 1, pipe.num_slots // 2):
        t = pipe.tiles(first=k, count=1)
        one = pipe.policy_loss(t, lp[t.elems], adv[t.rows], p, old[t.elems], kref[t.elems], H[t.elems],
                               weight[t.slots])
        assert abs(float(one[0][0]) - float(loss[k])) <= 2 * U * abs(float(loss[k]))
        assert torch.allclose(one[3], g[t.elems], rtol=4 * U, atol=0)
        pipe.preference_loss(t, lp[t.elems], torch.zeros(w.n, dtype=torch.int32, device="cuda"))
        pipe.check_losses()
    with pytest.raises(ValueError):
        pipe.tiles(first=0, count=pipe.num_slots + 1)


def test_chain_behind_a_stream_with_padding_views():
    """Sampler padding emits an identity twice: the first of its rows is paired."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(72)
    w = synth.window_from_ranks("loss_stream", [rng.integers(2, 60, 50), rng.integers(2, 60, 51)], 300)
    tok_off, toks, _ = synth.device_tensors(w, "cuda")
    perm = torch.from_numpy(rng.permutation(w.n).astype(np.int32)).cuda()
    ranks = 4
    win = odb.DeviceWindow(np.array([0, 25, 50, 75, w.n]), tok_off, toks)
    pipe = odb.StreamPipeline(win, perm, w.budget, buffer_size=16)
    pipe.plan()
    log(f"chain behind a stream: {pipe.num_slots} slots, {pipe.info['emitted_views']} views of {w.n}")
    assert pipe.info["emitted_views"] > w.n
    _chain(pipe, ranks, w.n, 61, 6)


def test_check_losses_raises_once():
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(73)
    w = synth.window_from_ranks("loss_check", [rng.integers(2, 30, 20)], 100)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")
    pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
    pipe.form()
    pipe.align()
    with pytest.raises(ValueError):
        pipe.tiles()
    pipe.collate()
    pipe.check_losses()
    t = pipe.tiles()
    lp = torch.zeros(t.num_elems, device="cuda")
    pair = torch.zeros(w.n, dtype=torch.int32, device="cuda")
    pipe.preference_loss(t, lp, pair)
    pipe.check_losses()
    pair[3] = 9
    pipe.preference_loss(t, lp, pair)
    with pytest.raises(odb.OdbError) as e:
        pipe.check_losses()
    assert e.value.status == odb.ODB_E_INVALID_DATA
    pipe.check_losses()


def test_pipeline_buffers_grow_behind_another_stream():
    """A larger run's call waits for one under way on another stream before it replaces its buffers."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(79)
    w = synth.window_from_ranks("loss_grow", [rng.integers(200, 600, 3000)], 40_000)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")
    pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
    pipe.form()
    pipe.align()
    pipe.collate()
    whole, part = pipe.tiles(), pipe.tiles(first=0, count=pipe.num_slots // 2)
    with pytest.raises(ValueError, match="labels"):
        pipe.tiles(pipe.outputs[1][:whole.num_elems - 1])
    gen = torch.Generator("cuda").manual_seed(79)
    lp = -torch.rand(whole.num_elems, generator=gen, device="cuda")
    adv = torch.randn(whole.num_rows, generator=gen, device="cuda")
    params = odb.PolicyParams(kl=0, reduce=1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = pipe.policy_loss(part, lp[part.elems], adv[part.rows], params, stream=side)
    b = pipe.policy_loss(whole, lp, adv, params)
    junk = torch.full((whole.num_elems,), -7.0, device="cuda")     # takes the memory that came free
    torch.cuda.synchronize()
    K = part.num_slots
    assert torch.equal(a[0], b[0][:K]) and torch.equal(a[2], b[2][:K])
    assert torch.equal(a[3], b[3][:part.num_elems]) and bool((junk == -7.0).all())
    pipe.check_losses()


def test_pipeline_losses_in_a_graph():
    """Both losses of a plan captured together and replayed on new inputs, eager work of another pipeline between."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(89)
    w = synth.window_from_ranks("loss_graph", [rng.integers(2, 300, 200), rng.integers(2, 300, 150)], 4000)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")

    def make():
        pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
        pipe.form()
        pipe.align()
        pipe.collate()
        return pipe, pipe.tiles()
    (pipe, t), (plain, u) = make(), make()
    pair = torch.zeros(w.n, dtype=torch.int32, device="cuda")
    pair[0:300:2] = torch.arange(1, 300, 2, dtype=torch.int32, device="cuda") + 1
    pair[1:300:2] = -(torch.arange(0, 300, 2, dtype=torch.int32, device="cuda") + 1)
    params = odb.PolicyParams(kl=2, reduce=1, kl_coef=0.1)
    gen = torch.Generator("cuda").manual_seed(89)
    draw = lambda: [-torch.rand(t.num_elems, generator=gen, device="cuda") * 3 for _ in range(3)] + \
        [torch.randn(t.num_rows, generator=gen, device="cuda")]
    lp, old, kref, adv = draw()
    call = lambda p, tiles, a: (p.policy_loss(tiles, a[0], a[3], params, a[1], a[2]) +
                                p.preference_loss(tiles, a[0], pair, ref_logprob=a[2]))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(pipe, t, (lp, old, kref, adv))
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = call(pipe, t, (lp, old, kref, adv))
    for _ in range(4):
        new = draw()
        for a, b in zip((lp, old, kref, adv), new):
            a.copy_(b)
        want = call(plain, u, new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert (a is None and b is None) or torch.equal(a, b)
    pipe.check_losses()
    plain.check_losses()
