"""The loss operators on the GPU where terms are far from ordinary: log ratios that pass fp32's exact
integers, NaN, terms that cancel or nearly overflow, weights that are not finite.

Tolerances count roundings of fp32 (U = 2^-24 relative each)."""
import math

import numpy as np
import pytest

from _losses import IGNORE, U, Plan
from test_gpu_losses import _policy_params, _policy_run, _preference_run, _tiles, _torch

pytestmark = pytest.mark.gpu

# one launch of one block, and the passes
SIZES = pytest.mark.parametrize("groups", [[[9, 40]], [[9, 40], [64] * 90]], ids=["one", "passes"])


def _dev(x):
    return _torch().from_numpy(np.ascontiguousarray(x)).cuda()


# ------------------------------------------------------------------------- policy loss
@SIZES
def test_slope_of_far_kl_terms(groups):
    """1 - exp(-x) of the exponential KL term where x is far larger than it, up to a reference of no probability."""
    torch = _torch()
    plan = Plan(groups)
    xs = np.array([0.0, 1e-3, -1e-3, 0.7, -0.7, 1.4, -1.4, 1.5, -1.5, 1.6, -1.6, 4.0, -4.0, 16.0, -16.0, 100.0, -80.0,
                   1e8, 16777218.0, 3e38, math.inf])
    lp = np.full(plan.E, -1.0, np.float32)
    with np.errstate(over="ignore"):
        kref = (lp - np.resize(xs, plan.E)).astype(np.float32)
    x = lp.astype(np.float64) - kref
    slope, power = -np.expm1(-x), np.exp(-x)
    # x is rounded once (U |x|), which moves the power by as much of itself; the power adds 8 of its own and
    # the difference one.  Below 3/2 the term is a series of which the slope is x less the term: 13 steps of
    # Horner's rule on terms of a sum of at most exp(|x|) - 1 - |x|, and a difference.
    moved = np.where(np.isinf(x), 0.0, np.abs(np.where(np.isinf(x), 0.0, x)) * power)
    a = np.minimum(np.abs(x), 1.5)
    series = np.where(np.abs(x) < 1.5, 2 * (np.expm1(a) - a) * 2, 8 * power)
    bound = U * (moved + series + 2 * np.abs(slope))
    adv = np.zeros(plan.R, np.float32)
    tiles = _tiles(plan, np.ones(plan.E, np.int32), 0, 0, 0)
    for reduce in range(3):
        out, status = _policy_run(tiles, plan, _policy_params(dict(kl=3, reduce=reduce, kl_coef=1.0, loss_scale=1.0)),
                                  _dev(lp), _dev(lp), _dev(kref), None, _dev(adv), None, extra=0)
        assert int(status.item()) == 0
        slot = plan.slot_of_row[plan.row_of]
        size = (plan.tile_off[1:] - plan.tile_off[:-1])[slot].astype(np.float64)
        w = 1.0 / size if reduce < 2 else np.ones(plan.E)        # every row of a slot is as long
        got = out["grad"].double().cpu().numpy()
        bad = ~(np.abs(got - w * slope) <= w * (bound + 2 * U * np.abs(slope)))
        assert not bad.any(), (reduce, x[bad][:8], got[bad][:8] / w[bad][:8], slope[bad][:8])


@SIZES
@pytest.mark.parametrize("reduce", range(3))
def test_terms_of_both_signs_in_one_group(groups, reduce):
    """Advantages per token whose large ones cancel, side by side: the small ones are what is left."""
    plan = Plan(groups)
    adv = np.resize(np.array([2.0 ** 24, 1, -2.0 ** 24, 1], np.float32), plan.E)
    n = (plan.tile_off[1:] - plan.tile_off[:-1])
    slot = plan.slot_of_row[plan.row_of]
    lp = np.full(plan.E, -1.0, np.float32)
    tiles = _tiles(plan, np.ones(plan.E, np.int32), 0, 0, 0)
    p = _policy_params(dict(kl=0, reduce=reduce, token_advantage=1, loss_scale=1.0))
    out, status = _policy_run(tiles, plan, p, _dev(lp), _dev(lp), None, None, _dev(adv), None, extra=0)
    assert int(status.item()) == 0
    total = -np.bincount(slot, weights=adv.astype(np.float64), minlength=plan.K)
    mags = np.bincount(slot, weights=np.abs(adv).astype(np.float64), minlength=plan.K)
    w = 1.0 / n if reduce < 2 else np.ones(plan.K)
    # weights and sums of 64 bits, each step at most 2^-53 of the sum of magnitudes, one rounding to fp32
    lost = 2.0 ** -52 * w * mags * (2 + n)
    assert np.all(np.abs(out["loss"].double().cpu().numpy() - w * total) <= U * np.abs(w * total) + lost)
    assert np.all(np.abs(out["means"][:, 0].double().cpu().numpy() - w * total) <= U * np.abs(w * total) + lost)


def test_linear_kl_terms_that_nearly_cancel():
    """Log ratios of few bits, so that every term is exact: what is left of terms a million times larger is
    rounded once, in every reduction."""
    rng = np.random.default_rng(67)
    for lens in ([3, 5, 7, 11], [int(v) for v in rng.integers(1, 90, 40)], [int(v) for v in rng.integers(100, 900, 40)]):
        plan = Plan([lens])
        y = plan.labels(rng)
        on = plan.counted(y, 0)
        x = rng.integers(-4096, 4097, plan.R) / 1024.0
        count = np.array([on[plan.row_of == r].sum() for r in range(plan.R)])
        for reduce, weight in ((0, count / count.sum()), (1, np.full(plan.R, 1 / plan.R)), (2, count.astype(np.float64))):
            # the last row's log ratio takes back the others', up to its own step
            x[-1] = np.round(-(x[:-1] * weight[:-1]).sum() / weight[-1] * 1024) / 1024
            kref = np.where(on, -x[plan.row_of], 0).astype(np.float32)
            tiles = _tiles(plan, y, 0, 0, 0)
            p = _policy_params(dict(kl=1, reduce=reduce, kl_coef=1.0, loss_scale=1.0))
            zero = np.zeros(plan.E, np.float32)
            out, _ = _policy_run(tiles, plan, p, _dev(zero), None, _dev(kref), None, _dev(np.zeros(plan.R, np.float32)),
                                 None, extra=0)
            want = (x * weight).sum()
            lost = 1e-15 * (np.abs(x) * weight).sum() * plan.E
            assert abs(float(out["loss"]) - want) <= U * abs(want) + lost, (plan.E, reduce, float(out["loss"]), want)
            assert abs(float(out["means"][0, 1]) - want) <= U * abs(want) + lost, (plan.E, reduce)


@SIZES
@pytest.mark.parametrize("reduce", [0, 1])
def test_means_of_terms_near_the_largest(groups, reduce):
    """KL terms, ratios and entropies of up to 2e38 have a mean."""
    plan = Plan(groups)
    n = plan.tile_off[1:] - plan.tile_off[:-1]
    slot = plan.slot_of_row[plan.row_of]
    d = np.resize(np.array([88.0, 87.5, 88.2, 88.0, 87.9], np.float32), plan.E)
    lp = np.zeros(plan.E, np.float32)
    H = np.full(plan.E, 2e38, np.float32)
    tiles = _tiles(plan, np.ones(plan.E, np.int32), 0, 0, 0)
    p = _policy_params(dict(kl=3, reduce=reduce, kl_coef=0.0, loss_scale=1.0, clip_high=math.inf))
    out, _ = _policy_run(tiles, plan, p, _dev(lp), _dev(-d), _dev(d), _dev(H), _dev(np.zeros(plan.R, np.float32)), None,
                         extra=0)
    mean = lambda v: np.bincount(slot, weights=v, minlength=plan.K) / n
    want = np.stack([mean(np.exp(d.astype(np.float64)) - 1 - d), mean(H.astype(np.float64)),
                     mean(np.exp(d.astype(np.float64)))], 1)
    got = out["means"][:, 1:].double().cpu().numpy()
    # the power of an argument that is exact: 8 roundings, a few for the sums
    assert np.all(np.abs(got - want) <= 16 * U * want), (got, want)


@SIZES
@pytest.mark.parametrize("reduce", range(3))
def test_tokens_that_do_not_count_beside_weights_that_are_not_finite(groups, reduce):
    rng = np.random.default_rng(3)
    plan = Plan(groups)
    y = plan.labels(rng, 0.6)
    on = plan.counted(y, 1)
    assert on.any() and not on.all()
    lp = np.where(on, -1.0, np.nan).astype(np.float32)
    H = np.where(on, 1.0, np.nan).astype(np.float32)
    adv = np.ones(plan.R, np.float32)
    tiles = _tiles(plan, y, 1, 0, 0)
    for kl in range(4):
        p = _policy_params(dict(kl=kl, reduce=reduce, kl_coef=0.5, entropy_coef=0.1, loss_scale=1e30))
        for w in (math.inf, math.nan, 1e30):
            out, _ = _policy_run(tiles, plan, p, _dev(lp), None, _dev(lp) if kl else None, _dev(H), _dev(adv),
                                 _dev(np.full(plan.K, w)), extra=0)
            for k in ("grad", "grad_ent"):
                assert np.all(out[k].cpu().numpy()[~on] == 0), (kl, w, k)
                assert not np.isfinite(out[k].cpu().numpy()[on]).any(), (kl, w, k)


# --------------------------------------------------------------------- preference loss
@pytest.mark.parametrize("rows", [8, 40, 600], ids=["one", "few", "many"])
@pytest.mark.parametrize("by_id", [False, True])
@pytest.mark.parametrize("kind", range(3))
def test_pairs_without_a_number(rows, by_id, kind):
    """A NaN among a pair's log-probabilities, or no probability on either side: the pair's loss and gradients
    are NaN, and the total's; the other pairs keep theirs."""
    torch = _torch()
    plan = Plan([[40] * rows])
    y = np.ones(plan.E, np.int32)
    rng = np.random.default_rng(rows)
    pair = np.zeros(plan.R, np.int32)
    pair[0::2], pair[1::2] = np.arange(1, plan.R, 2) + 1, -(np.arange(0, plan.R, 2) + 1)
    p = dict(kind=kind, normalize=0, beta=0.1, margin=0.1, label_smoothing=0.0, loss_scale=1.0)
    tiles = _tiles(plan, y, 0, 0, 0)
    ids = _dev(np.arange(plan.R, dtype=np.int32)) if by_id else None
    base = (-rng.random(plan.E)).astype(np.float32)
    good, _ = _preference_run(tiles, plan, p, _dev(base), None, ids, _dev(pair), 0, 0)
    for c, values in ((4, {4: math.nan}), (2, {3: math.nan}), (6, {6: -math.inf, 7: -math.inf})):
        lp = base.copy()
        for r, v in values.items():
            lp[np.nonzero(plan.row_of == r)[0][17]] = v
        out, status = _preference_run(tiles, plan, p, _dev(lp), None, ids, _dev(pair), 0, 0)
        assert int(status.item()) == 0
        assert math.isnan(out["loss"].item()), (c, kind)
        assert out["counts"][0].item() == plan.R // 2
        mine = np.isin(np.arange(plan.R), (c, c + 1))
        row_loss, grad = out["row_loss"].cpu().numpy(), out["grad"].cpu().numpy()
        assert math.isnan(row_loss[c]) and row_loss[c + 1] == 0
        assert np.array_equal(row_loss[~mine], good["row_loss"].cpu().numpy()[~mine])
        at = mine[plan.row_of]
        assert np.isnan(grad[at]).all() and np.array_equal(grad[~at], good["grad"].cpu().numpy()[~at])


# ------------------------------------------------------------------ arrays that contradict each other
def _broken(plan, field, at, value):
    bad = Plan([[1]])
    for name in ("rows", "maxlen", "row_off", "tile_off"):
        setattr(bad, name, getattr(plan, name).copy())
    getattr(bad, field)[at] = value
    bad.R, bad.E, bad.K = plan.R, plan.E, plan.K
    return bad


BROKEN = {
    # name: (groups, offsets that fall or leave the arrays, slots whose rows do not fit their offsets)
    "one": ([[4, 6], [9], [3, 3, 3]], [("tile_off", 3, 5), ("tile_off", 3, -2), ("tile_off", 1, 10 ** 9), ("row_off", 3, 0)],
            [("rows", 1, 2), ("maxlen", 2, 4)]),
    "passes": ([[70] * 10] * 12, [("tile_off", 2, 1 << 40), ("tile_off", 2, 9000), ("tile_off", 2, -1),
                                  ("tile_off", 12, 700), ("tile_off", 12, -5), ("tile_off", 6, 0), ("row_off", 5, 0),
                                  ("row_off", 12, 1000), ("row_off", 12, 3), ("row_off", 1, 1 << 40)],
               [("rows", 3, 9), ("maxlen", 3, 71), ("rows", 0, -1), ("maxlen", 11, 0), ("rows", 11, 1 << 30)]),
    "many": ([[9] * 10] * 700, [("tile_off", 600, 0), ("row_off", 699, 1 << 50)], [("rows", 600, 9), ("maxlen", 0, 8)]),
}


@pytest.mark.parametrize("name", list(BROKEN))
def test_slots_that_contradict_each_other(name):
    """Whatever the workspace held: beside a slot whose rows do not fit the others have their numbers; with
    offsets out of order a slot has its numbers or none."""
    torch = _torch()
    groups, offsets, slots = BROKEN[name]
    plan = Plan(groups)
    rng = np.random.default_rng(7)
    y = plan.labels(rng, 0.3)
    on = plan.counted(y, 1)
    lp = np.where(on, -rng.random(plan.E), 0).astype(np.float32)
    old, kref = (np.where(on, lp + rng.normal(size=plan.E) * 0.1, 0).astype(np.float32) for _ in range(2))
    adv = rng.standard_normal(plan.R).astype(np.float32)
    pair = np.zeros(plan.R, np.int32)
    at = rng.permutation(plan.R)[:plan.R // 2 * 2]
    pair[at[0::2]], pair[at[1::2]] = at[1::2] + 1, -(at[0::2] + 1)
    pp = dict(kind=0, normalize=0, beta=0.2, margin=0.0, label_smoothing=0.0, loss_scale=1.0)
    slot_of = plan.slot_of_row[plan.row_of]
    good = [_policy_run(_tiles(plan, y, 1, 0, 0), plan, _policy_params(dict(kl=3, reduce=r)), _dev(lp), _dev(old),
                        _dev(kref), None, _dev(adv), None, extra=0)[0] for r in range(3)]
    fair, _ = _preference_run(_tiles(plan, y, 1, 0, 0), plan, pp, _dev(lp), _dev(kref), None, _dev(pair), 0, 0)
    for field, k, value in offsets + slots:
        tiles = _tiles(_broken(plan, field, k, value), y, 1, 0, 0)
        ordered = (field, k, value) in slots
        left = [torch.full((1 << 20,), fill, dtype=torch.uint8, device="cuda") for fill in (0x3f, 0x01)]
        for reduce in range(3):
            for ws in left:
                out, status = _policy_run(tiles, plan, _policy_params(dict(kl=3, reduce=reduce)), _dev(lp), _dev(old),
                                          _dev(kref), None, _dev(adv), None, extra=0, ws=ws)
                assert int(status.item()) != 0
                for key in ("loss", "means", "counts"):
                    got, want = out[key].cpu().numpy(), good[reduce][key].cpu().numpy()
                    if ordered:
                        want[k] = 0
                        assert np.array_equal(got, want), (field, k, value, reduce, key)
                    else:
                        whole = np.array([np.array_equal(g, w) for g, w in zip(got, want)])
                        none = np.array([not np.any(g) for g in got])
                        assert np.all(whole | none), (field, k, value, reduce, key, got)
                if ordered:
                    other = slot_of != k
                    assert np.array_equal(out["grad"].cpu().numpy()[other], good[reduce]["grad"].cpu().numpy()[other])
        for ids in (None, _dev(np.arange(plan.R, dtype=np.int32))):
            out, status = _preference_run(tiles, plan, pp, _dev(lp), _dev(kref), ids, _dev(pair), 0, 0, ws=left[0])
            assert int(status.item()) != 0
            got = {key: v.cpu().numpy() for key, v in out.items()}
            if not ordered:
                assert got["loss"][0] == 0 and not got["counts"].any()
                # rows behind the last offset are behind the run
                assert np.isin(got["row_loss"], (0, -3)).all() and np.isin(got["reward"], (0, -3)).all()
                continue
            lost = plan.slot_of_row == k
            partner = np.abs(pair.astype(np.int64)) - 1
            unpaired = lost | ((partner >= 0) & lost[partner])
            want = np.where(unpaired, 0, fair["row_loss"].cpu().numpy())
            assert np.array_equal(got["row_loss"], want)
            assert np.array_equal(got["reward"], np.where(lost, 0, fair["reward"].cpu().numpy()))
            assert got["counts"][0] == ((pair > 0) & ~unpaired).sum()
            total = want.astype(np.float64).sum()
            assert abs(got["loss"][0] - total) <= 2 * U * np.abs(want).sum()     # rows rounded once each, and the total
            at = ~lost[plan.row_of]
            grad = np.where(unpaired[plan.row_of], 0, fair["grad"].cpu().numpy())
            assert np.array_equal(got["grad"][at], grad[at])
        # nothing stays behind in the workspace
        tiles = _tiles(plan, y, 1, 0, 0)
        for reduce in range(3):
            out, status = _policy_run(tiles, plan, _policy_params(dict(kl=3, reduce=reduce)), _dev(lp), _dev(old),
                                      _dev(kref), None, _dev(adv), None, extra=0, ws=left[0])
            assert int(status.item()) == 0
            assert all(v is None or torch.equal(v, good[reduce][key]) for key, v in out.items()), (field, k, value)
        out, status = _preference_run(tiles, plan, pp, _dev(lp), _dev(kref), None, _dev(pair), 0, 0, ws=left[0])
        assert int(status.item()) == 0 and all(torch.equal(v, fair[key]) for key, v in out.items()), (field, k, value)


# ------------------------------------------------------------------------- slots of many chunks
@pytest.mark.parametrize("reduce", range(3))
def test_one_slot_of_very_many_chunks(reduce):
    """2^28 elements in one slot: their numbers, in a time near that of as many in 256 slots (what each chunk
    adds up must not grow with its slot)."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    E, L = 1 << 28, 512
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    gen = torch.Generator("cuda").manual_seed(5)
    y = torch.randint(-130, 200, (E,), generator=gen, **i32).clamp_(min=IGNORE)       # 1 in 11 does not count
    y.view(-1, L)[::5] = IGNORE                                                        # rows in which nothing does
    lp = torch.rand(E, generator=gen, device="cuda") - 1
    grad = torch.empty(E, device="cuda")
    adv = torch.randn(E // L, generator=gen, device="cuda")
    on = (y != IGNORE).view(-1, L)
    on[:, 0] = False
    count = on.sum(1)
    took = {}
    for K in (256, 1):
        rows = E // L // K
        tiles = odb.Tiles(torch.full((K,), rows, **i32), torch.full((K,), L, **i32), torch.arange(K + 1, **i64) * rows,
                          torch.arange(K + 1, **i64) * rows * L, y, E // L)
        ws = torch.full((odb.odb_loss_workspace_size(tiles),), 0x7f, dtype=torch.uint8, device="cuda")
        loss, means, counts = torch.empty(K, device="cuda"), torch.empty(K, 4, device="cuda"), torch.empty(K, 4, **i64)
        call = lambda: odb.odb_policy_loss(tiles, odb.PolicyParams(reduce=reduce), lp, adv, loss, means, counts, ws,
                                           grad_logprob=grad)
        call()
        n = count.view(K, rows).sum(1)
        real = (count > 0).view(K, rows).sum(1)
        w = {0: 1.0 / n.double()[:, None].expand(K, rows), 2: torch.ones(K, rows, device="cuda").double(),
             1: 1.0 / (count.clamp(min=1).double().view(K, rows) * real[:, None])}[reduce]
        terms = -adv.double().view(K, rows) * w * count.view(K, rows)
        want, mag = terms.sum(1), terms.abs().sum(1)
        assert torch.equal(counts[:, 0], n)
        assert torch.all((loss.double() - want).abs() <= U * want.abs() + 1e-12 * mag)
        g = (-adv.double() * w.reshape(-1))                 # two roundings: the factor, the product
        assert torch.all((grad.view(-1, L)[:, 7].double() - g * on[:, 7]).abs() <= 2.01 * U * g.abs())
        assert torch.all(grad.view(-1, L)[~on] == 0)
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call()
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        took[K] = min(times)
    assert took[1] < 2 * took[256], took        # 1.3; with a sum per chunk over its whole slot 4 to 6
