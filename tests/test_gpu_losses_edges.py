"""The loss operators on the GPU where terms are far from ordinary: log ratios that pass fp32's exact
integers, NaN, terms that cancel or nearly overflow, weights that are not finite.

Tolerances count roundings of fp32 (U = 2^-24 relative each)."""
import math

import numpy as np
import pytest

import _losses as ref
from _losses import U, Plan
from test_gpu_losses import _pad, _policy_params, _policy_run, _preference_run, _tiles, _torch

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
