"""The distillation loss on the GPU against its definition in 64 bits: every divergence, support and reduction,
lists of every length, slots and rows across pieces and chunks, lists that end early or are empty, infinities
and NaN in places that do not count."""
import math

import numpy as np
import pytest

import _lists as ref
from _losses import IGNORE, U, Plan
from _parity import log

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _dev(v):
    return None if v is None else _torch().from_numpy(np.ascontiguousarray(v)).cuda()


def _lists(rng, E, k, near=0.7, short=0.3):
    """A teacher's and a student's log-probabilities of E lists: the likeliest first, some lists end early."""
    z = -np.cumsum(rng.exponential(0.5, (E, k)), -1)

    def part(z):
        m = z.max(-1, keepdims=True)
        return z - m - np.log(np.exp(z - m).sum(-1, keepdims=True)) + np.log(rng.uniform(0.6, 0.999, (E, 1)))

    t = part(z).astype(np.float32)
    s = part(z + near * rng.standard_normal((E, k))).astype(np.float32)
    ends = np.where(rng.random(E) < short, rng.integers(0, k + 1, E), k)
    none = np.arange(k)[None] >= ends[:, None]
    t[none] = -math.inf
    s[none] = np.where(rng.random(int(none.sum())) < 0.5, math.nan, math.inf).astype(np.float32)
    return t, s


class Run:
    def __init__(self, plan, labels, t, s, k, params, slot_weight=None, shift=1, grad=True, extra=0, stream=None):
        import paper_2606_19989_amd as odb
        torch = _torch()
        self.base = plan
        self.tiles = odb.Tiles(_dev(plan.rows), _dev(plan.maxlen), _dev(plan.row_off), _dev(plan.tile_off),
                               _dev(labels), plan.R, shift)
        self.k, self.params = k, params
        self.t, self.s, self.w = _dev(t), _dev(s), _dev(slot_weight)
        K, E = self.tiles.num_slots, self.tiles.num_elems
        self.loss = torch.full((K,), 7.0, device="cuda")
        self.mean = torch.full((K,), 7.0, device="cuda")
        self.count = torch.full((K,), 7, dtype=torch.int64, device="cuda")
        self.grad = torch.full((E, k), 7.0, device="cuda") if grad else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.full((odb.odb_distill_workspace_size(self.tiles, k),), 0xa5, dtype=torch.uint8, device="cuda")

    def __call__(self, stream=None):
        import paper_2606_19989_amd as odb
        odb.odb_distill_loss(self.tiles, self.params, self.s, self.t, self.loss, self.mean, self.count, self.ws,
                             slot_weight=self.w, grad_student=self.grad, status=self.status, stream=stream)

    def numpy(self):
        _torch().cuda.synchronize()
        f = lambda v: None if v is None else v.cpu().numpy()
        return f(self.loss).astype(np.float64), f(self.mean).astype(np.float64), f(self.count), \
            None if self.grad is None else f(self.grad).astype(np.float64)


def _check(run, plan, labels, t, s, k, p, slot_weight, shift):
    loss, mean, count, grad, e_mean, e_grad = ref.distill(plan, labels, s.astype(np.float64), t.astype(np.float64), k,
                                                          p["kind"], p["support"], p["reduce"], p.get("mix", 0.5),
                                                          slot_weight, p.get("loss_scale", 1.0), shift)
    g_loss, g_mean, g_count, g_grad = run.numpy()
    assert int(run.status.item()) == 0
    assert np.array_equal(g_count, count)
    tol = U * (e_mean + 2 * np.abs(mean)) + 1e-300
    assert np.all(np.abs(g_mean - mean) <= tol), (np.abs(g_mean - mean) / tol).max()
    sw = p.get("loss_scale", 1.0) * (np.ones(plan.K) if slot_weight is None else slot_weight)
    assert np.all(np.abs(g_loss - loss) <= np.abs(sw) * tol + 2 * U * np.abs(loss))
    assert np.all(g_mean[count == 0] == 0) and np.all(g_loss[count == 0] == 0)
    if g_grad is not None:
        on = plan.counted(labels, shift)
        assert np.all(g_grad[~on] == 0) and np.all(g_grad[t == -math.inf] == 0)
        # products with a factor rounded to 32 bits; probabilities below the normal numbers may be 0
        tol = U * (e_grad + 4 * np.abs(grad)) + 2.0 ** -115
        err = np.abs(g_grad - grad)
        assert np.all(err <= tol), (err / tol).max()


SMALL = [[5, 3, 4], [], [1], [7, 7], [1, 1, 1]]
KS = [1, 2, 3, 4, 5, 7, 8, 13, 16, 17, 27, 32, 33, 63, 64, 65, 100, 127, 128]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("support", [0, 1, 2])
def test_every_length_of_list(kind, support):
    """One launch of one block where entries are few, the passes where they are many."""
    import paper_2606_19989_amd as odb
    for k in KS:
        log(f"distill kind {kind} support {support} k {k}")
        rng = np.random.default_rng(k)
        for groups in (SMALL, [[40, 33], [90] * 3, [1] * 7, [], [300]] * 2):
            plan = Plan(groups, base=(3, 17))
            y = plan.labels(rng, prompt=0.5, empty=0.2)
            t, s = _lists(rng, plan.E, k)
            off = ~plan.counted(y, 1)
            t[off], s[off] = math.nan, math.inf         # nothing of a token that does not count is read
            p = dict(kind=kind, support=support, reduce=k % 3, mix=0.3, loss_scale=2.5)
            w = rng.random(plan.K)
            run = Run(plan, y, t, s, k, odb.DistillParams(**p), w)
            run()
            _check(run, plan, y, np.where(off[:, None], -math.inf, t), np.where(off[:, None], 0.0, s), k, p, w, 1)


@pytest.mark.parametrize("reduce", [0, 1, 2])
@pytest.mark.parametrize("shape", ["one tile", "tiles", "single columns", "long rows", "idle ranks"])
def test_slots_and_rows_across_pieces(shape, reduce):
    import paper_2606_19989_amd as odb
    log(f"distill {shape} reduce {reduce}")
    rng = np.random.default_rng(len(shape) + reduce)
    groups = {"one tile": [list(rng.integers(60, 70, 100))], "tiles": [list(rng.integers(1, 90, n)) for n in rng.integers(1, 30, 60)],
              "single columns": [[1] * 5000, [2] * 1000], "long rows": [[12000, 11000], [9000]],
              "idle ranks": [[]] * 5000 + [[30] * 20] + [[]] * 3000 + [[7] * 99] + [[]] * 2}[shape]
    plan = Plan(groups)
    for shift in (0, 1):
        y = plan.labels(rng, prompt=0.8, empty=0.3)
        k = 3
        t, s = _lists(rng, plan.E, k)
        p = dict(kind=0, support=1, reduce=reduce, loss_scale=0.5)
        w = rng.random(plan.K)
        run = Run(plan, y, t, s, k, odb.DistillParams(**p), w, shift=shift)
        run()
        _check(run, plan, y, t, s, k, p, w, shift)
        first = [v.copy() for v in run.numpy()]
        run()
        assert all(np.array_equal(a, b) for a, b in zip(first, run.numpy())), "not the same bit for bit"


@pytest.mark.parametrize("reduce", [0, 1, 2])
def test_many_short_rows(reduce):
    """A million elements in rows of 1 to 5, with few entries: thousands of rows in a piece, rows cut by its ends."""
    import paper_2606_19989_amd as odb
    rng = np.random.default_rng(11)
    plan = Plan([[1] * 100_001, [5] * 70_003, [], [3] * 120_007, [2] * 70_001, [40_000] * 2])
    log(f"distill: {plan.E} elements in {plan.R} rows")
    y = plan.labels(rng, prompt=0.9, empty=0.2)
    k = 2
    t, s = _lists(rng, plan.E, k)
    w = rng.random(plan.K)
    run = Run(plan, y, t, s, k, odb.DistillParams(reduce=reduce, loss_scale=2.0), w)
    run()
    loss, mean, count, grad = run.numpy()
    assert int(run.status.item()) == 0
    on = plan.counted(y, 1)
    there = t != -math.inf
    t64, s64 = np.where(there, t, 0.0).astype(np.float64), np.where(there, s, 0.0).astype(np.float64)
    p = np.where(there, np.exp(t64), 0.0)
    D = (p * (t64 - s64)).sum(-1)
    slot = plan.slot_of_row[plan.row_of]
    n = np.bincount(slot[on], minlength=plan.K)
    per_row = np.bincount(plan.row_of[on], minlength=plan.R)
    rows = np.bincount(plan.slot_of_row[per_row > 0], minlength=plan.K)
    with np.errstate(divide="ignore"):
        f = [1.0 / n[slot], 1.0 / (per_row[plan.row_of] * rows[slot]), np.ones(plan.E)][reduce]
    f = np.where(on, f, 0.0)
    assert np.array_equal(count, n)
    size = (p * (np.abs(t64) + np.abs(s64) + 4) * (1 + np.abs(t64 - s64))).sum(-1)      # as in the oracle's bounds
    want = np.bincount(slot, weights=f * D, minlength=plan.K)
    tol = U * np.bincount(slot, weights=f * (4 * size + 12 * np.abs(D)), minlength=plan.K) + 2 * U * np.abs(want)
    assert np.all(np.abs(mean - want) <= tol)
    assert np.all(np.abs(loss - 2 * w * want) <= 2 * w * tol + 2 * U * np.abs(2 * w * want))
    want = -(2 * w[slot] * f)[:, None] * p
    assert np.all(np.abs(grad - want) <= U * np.abs(want) * (4 * (np.abs(t64) + np.abs(s64) + 4) + 4) + 2.0 ** -115)


def test_nothing_counts_and_no_slots():
    import paper_2606_19989_amd as odb
    plan = Plan([[4, 3], [], [2]])
    y = np.full(plan.E, IGNORE, np.int32)
    t = s = np.full((plan.E, 4), math.nan, np.float32)
    for reduce in range(3):
        run = Run(plan, y, t, s, 4, odb.DistillParams(reduce=reduce), np.full(plan.K, math.inf))
        run()
        loss, mean, count, grad = run.numpy()
        assert not loss.any() and not mean.any() and not count.any() and not grad.any()
    plan = Plan([[], []])
    run = Run(plan, np.zeros(0, np.int32), np.zeros((0, 4), np.float32), np.zeros((0, 4), np.float32), 4, odb.DistillParams())
    run()
    assert all(not v.any() for v in run.numpy())
    Run(Plan([]), np.zeros(0, np.int32), np.zeros((0, 4), np.float32), np.zeros((0, 4), np.float32), 4,
        odb.DistillParams())()


@pytest.mark.parametrize("n", [3, 3000])
def test_probabilities_of_zero_and_one(n):
    """Students that give a listed token nothing, teachers sure of one token, lists that hold everything."""
    import paper_2606_19989_amd as odb
    plan = Plan([[5] * n])
    rng = np.random.default_rng(2)
    y = plan.labels(rng)
    E = plan.E
    sure = np.array([0.0, -200.0, -math.inf], np.float32)
    part = np.log([0.5, 0.3, 0.1]).astype(np.float32)
    none = np.array([-math.inf, -1.0, -2.0], np.float32)
    low = np.array([-120.0, -1.0, -1.0], np.float32)

    def one(t, s, **p):
        p = {**dict(kind=0, support=0, reduce=0), **p}
        T, S = np.tile(t, (E, 1)), np.tile(s, (E, 1))
        run = Run(plan, y, T, S, 3, odb.DistillParams(**p), shift=0)
        run()
        return run, T, S, p

    # a forward divergence is infinite where the student gives nothing, and its slope is not
    run, *_ = one(part, none)
    loss, mean, count, grad = run.numpy()
    assert mean[0] == math.inf and np.isfinite(grad).all()
    run, *_ = one(part, none, kind=2)
    loss, mean, count, grad = run.numpy()
    assert np.isfinite(mean).all() and np.isfinite(grad).all() and np.all(grad[:, 0] == 0)
    for kind in (0, 1, 2):
        for support in (0, 1, 2):
            cases = [(sure, part), (part, sure[:2].tolist() + [-3.0])]
            if kind:
                cases += [(part, none), (part, low)]
            for t, s in cases:
                log(f"  kind {kind} support {support} {t} {s}")
                run, T, S, p = one(np.asarray(t, np.float32), np.asarray(s, np.float32), kind=kind, support=support, mix=0.7)
                with np.errstate(all="ignore"):
                    _check(run, plan, y, T, S, 3, p, None, 0)


def test_a_nan_stays():
    import paper_2606_19989_amd as odb
    plan = Plan([[4, 4], [3]])
    rng = np.random.default_rng(3)
    y = np.zeros(plan.E, np.int32)
    for kind in range(3):
        for support in range(3):
            for of in ("t", "s"):
                t, s = _lists(rng, plan.E, 6, short=0.0)
                (t if of == "t" else s)[2, 1] = math.nan
                run = Run(plan, y, t, s, 6, odb.DistillParams(kind=kind, support=support), shift=0)
                run()
                loss, mean, count, grad = run.numpy()
                assert math.isnan(mean[0]) and math.isnan(loss[0]) and math.isfinite(mean[1]), (kind, support, of)
                # the forward divergence of entries as they are has the slope -p, whatever the student gives
                assert np.isnan(grad[2, 1]) == (kind != 0 or support != 0 or of == "t")
                assert np.isfinite(grad[np.arange(plan.E) != 2]).all()


@pytest.mark.parametrize("n", [3, 900])
def test_no_entry_has_gradient_0_beside_weights_that_are_not_finite(n):
    import paper_2606_19989_amd as odb
    plan = Plan([[5] * n, [4]])
    rng = np.random.default_rng(8)
    y = plan.labels(rng)
    t, s = _lists(rng, plan.E, 6, short=0.5)
    on = plan.counted(y, 1)
    for support in range(3):
        for w in (math.inf, math.nan):
            run = Run(plan, y, t, s, 6, odb.DistillParams(kind=1, support=support), np.array([w, 1.0]))
            run()
            loss, mean, count, grad = run.numpy()
            assert not math.isfinite(loss[0]) and math.isfinite(loss[1]) and np.isfinite(mean).all()
            assert np.all(grad[~on] == 0) and np.all(grad[t == -math.inf] == 0)


def test_without_gradient_and_weights():
    import paper_2606_19989_amd as odb
    rng = np.random.default_rng(4)
    for groups in ([[9, 8]], [[200] * 30]):
        plan = Plan(groups)
        y = plan.labels(rng, prompt=0.4)
        t, s = _lists(rng, plan.E, 12)
        a = Run(plan, y, t, s, 12, odb.DistillParams(kind=1))
        b = Run(plan, y, t, s, 12, odb.DistillParams(kind=1), grad=False)
        a()
        b()
        assert all(np.array_equal(x, z) for x, z in zip(a.numpy()[:3], b.numpy()[:3]))


@pytest.mark.parametrize("many", [False, True])
def test_contradicting_slots_are_reported(many):
    """A slot whose rows do not fit its offsets counts nothing; the others are as without it."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(5)
    plan = Plan([[30] * 3, [20] * 4, [10] * 5] * (20 if many else 1))
    y = plan.labels(rng)
    t, s = _lists(rng, plan.E, 8)
    for reduce in range(3):
        good = Run(plan, y, t, s, 8, odb.DistillParams(reduce=reduce))
        good()
        loss, mean, count, grad = good.numpy()
        bad = Run(plan, y, t, s, 8, odb.DistillParams(reduce=reduce))
        bad.tiles.keep[1][1] = 21
        bad()
        bl, bm, bc, bg = bad.numpy()
        assert int(bad.status.item()) != 0
        assert bl[1] == 0 and bm[1] == 0 and bc[1] == 0
        keep = np.arange(plan.K) != 1
        assert np.array_equal(bl[keep], loss[keep]) and np.array_equal(bc[keep], count[keep])
        a, b = plan.tile_off[1], plan.tile_off[2]
        assert np.all(bg[a:b] == 7.0)
        assert np.array_equal(np.delete(bg, np.s_[a:b], 0), np.delete(grad, np.s_[a:b], 0))
    # offsets that fall: any slot may count nothing, nothing is read or written outside
    worse = Run(plan, y, t, s, 8, odb.DistillParams(reduce=1))
    worse.tiles.keep[3][2] = -5
    worse()
    torch.cuda.synchronize()
    assert int(worse.status.item()) != 0


def test_elements_behind_the_last_slot_stay():
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(6)
    for groups in ([[9, 8]], [[100] * 60]):
        plan = Plan(groups)
        y = np.concatenate([plan.labels(rng), np.zeros(777, np.int32)])
        t, s = _lists(rng, plan.E + 777, 5)
        run = Run(plan, y, t, s, 5, odb.DistillParams())
        run()
        assert np.all(run.numpy()[3][plan.E:] == 7.0)
        short = Run(plan, y[:plan.E], t[:plan.E], s[:plan.E], 5, odb.DistillParams())
        short()
        assert np.array_equal(run.numpy()[0], short.numpy()[0])


def test_gradient_against_differences():
    import paper_2606_19989_amd as odb
    rng = np.random.default_rng(7)
    plan = Plan([[3, 2], [2]])
    y = plan.labels(rng)
    for kind in range(3):
        for support in range(3):
            t, s = _lists(rng, plan.E, 5, short=0.2)
            s[t == -math.inf] = 0.0
            make = lambda s: Run(plan, y, t, s, 5, odb.DistillParams(kind=kind, support=support, reduce=2), shift=0)
            run = make(s)
            run()
            grad = run.numpy()[3]
            h = 2.0 ** -6
            for e, j in [(0, 0), (1, 2), (4, 1)]:
                if t[e, j] == -math.inf:
                    continue
                v = []
                for d in (h, -h):
                    moved = s.copy()
                    moved[e, j] += np.float32(d)
                    r = make(moved)
                    r()
                    v.append(r.numpy()[0].sum())
                # third derivatives of these terms stay below 40, values of about 10 are right to a few U each
                assert abs((v[0] - v[1]) / (2 * h) - grad[e, j]) <= 40 * h * h / 6 + 64 * U * 10 / h, (kind, support, e, j)
