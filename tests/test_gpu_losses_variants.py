"""Every variant that the loss operators choose by sizes and options against the definitions in 64 bits: threads
of a position by the bytes of its logits, and the policy loss's passes by KL term, reduction and entropies, in
runs of a few and of many chunks.

Tolerances count roundings of fp32 (U = 2^-24 relative each) and of the output's type."""
import math

import numpy as np
import pytest

import _losses as ref
import test_gpu_losses as base
from _losses import IGNORE, U, Plan
from _parity import log

pytestmark = pytest.mark.gpu

# More positions than twice the compute units, so that threads go by the bytes of a row alone:
# rows, cols, V, dtype, shift, scale, pad, entropy
MANY_POSITIONS = [
    # 1 to 2 KB
    (40, 15, 257, "fp32", 1, 1.0, 0, True), (1, 601, 300, "fp32", 0, 1.0, 3, False), (40, 15, 512, "fp32", 1, 0.5, 0, True),
    (60, 9, 513, "bf16", 1, 1.0, 0, False), (40, 15, 600, "bf16", 1, 1.5, 1, True), (40, 14, 1023, "bf16", 0, 1.0, 0, True),
    (70, 8, 1024, "bf16", 1, 1.0, 0, False), (60, 9, 513, "fp16", 1, 1.0, 2, True), (40, 15, 1000, "fp16", 1, 1.0, 0, False),
    (20, 27, 1021, "fp16", 1, 0.75, 0, True),
    # below, and above
    (40, 15, 255, "fp32", 1, 1.0, 0, True), (40, 15, 512, "bf16", 1, 1.0, 0, True), (40, 15, 1031, "bf16", 1, 1.0, 0, True),
    (40, 14, 2051, "fp32", 1, 1.0, 0, True), (20, 27, 5003, "fp16", 1, 1.0, 0, True), (30, 18, 10007, "bf16", 1, 1.0, 0, False),
]


@pytest.mark.parametrize("case", MANY_POSITIONS, ids=str)
def test_token_logprobs_of_many_positions(case):
    assert case[0] * case[1] > 2 * 256
    base.test_token_logprobs_and_gradient(case)


def _policy64(m, plan, y, p, lp, old, kref, H, adv, w):
    """Every output of the policy loss in 64 bits, shift 1, and bounds on the fp32 roundings of each.

    A power is off by the rounding of its argument d (U |d|) and 8 of its own; the policy term adds a product.  A
    rounding of the log ratio x moves a KL term by |x| |slope|; the exponential one adds a series of 13 steps
    whose terms add up to exp(|x|) - 1 - |x| below 3/2, a power and two differences above."""
    torch = base._torch()
    zero = torch.zeros((), dtype=torch.float64, device=y.device)
    on = (y != IGNORE) & (m.col >= 1)
    of = lambda v: torch.where(on, v.double(), zero)
    K = plan.K
    n_slot, n_row = m.sum(on, m.by_slot), m.sum(on, m.by_row)
    n_rows = m.sum(n_row > 0, m.rows_of_slot)
    weight = of([lambda: 1 / n_slot[m.slot], lambda: 1 / (n_row[m.row] * n_rows[m.slot]),
                 lambda: torch.ones_like(m.slot)][p["reduce"]]())
    A = of(adv if p["token_advantage"] else adv[m.row])
    d, kc, ec = of(lp) - of(old), p["kl_coef"], p["entropy_coef"]
    r = d.exp()
    low = on & (A < 0) & (d < math.log1p(-p["clip_low"]))
    high = on & (A > 0) & (d > math.log1p(p["clip_high"]))
    dual = on & (A < 0) & (d > (math.log(p["dual_clip"]) if p["dual_clip"] else math.inf))
    clipped = low | high | dual
    policy = -torch.where(high, 1 + p["clip_high"], torch.where(low, 1 - p["clip_low"],
                                                                torch.where(dual, p["dual_clip"], r))) * A
    e_policy = U * torch.where(clipped, 3.0, 12.0 + d.abs()) * policy.abs()
    v_slope, e_v = torch.where(clipped, zero, policy), torch.where(clipped, zero, e_policy)
    x = of(lp) - of(kref) if p["kl"] else torch.zeros_like(d)
    a, far = x.abs(), x.abs() >= 1.5
    if p["kl"] == 3:
        kl, slope, power = torch.expm1(-x) + x, -torch.expm1(-x), torch.exp(-x)
        series = 8 * (torch.expm1(a.clamp(max=1.5)) - a.clamp(max=1.5))
        e_kl = U * (a * slope.abs() + torch.where(far, 8 * power + 2 * (a + 1), series))
        e_slope = U * (a * power + torch.where(far, 8 * power, series) + 2 * slope.abs())
    else:
        kl, slope = [(x * 0, x * 0), (x, x * 0 + 1), (x * x / 2, x)][p["kl"]]
        e_kl, e_slope = 4 * U * kl.abs(), 2 * U * slope.abs()
    ent = of(H) if H is not None else torch.zeros_like(d)
    scale = p["loss_scale"] * w
    mean = lambda v: m.sum(weight * v, m.by_slot)
    means = torch.stack([mean(policy), mean(kl), mean(ent), mean(r)], 1)
    e_means = torch.stack([mean(e_policy), mean(e_kl), mean(ent) * 0, mean(U * (10 + d.abs()) * r)], 1)
    mags = torch.stack([mean(v.abs()) for v in (policy, kl, ent, r)], 1)
    loss = scale * (means[:, 0] + kc * means[:, 1] - ec * means[:, 2])
    factor = weight * scale[m.slot]
    grad = factor * (v_slope + kc * slope)
    return dict(
        on=on, loss=loss, e_loss=scale * (e_means[:, 0] + abs(kc) * e_means[:, 1] + 1e-12 * mags.sum(1)) + U * loss.abs(),
        means=means, e_means=e_means + U * means.abs() + 1e-12 * mags,
        counts=torch.stack([m.sum(v, m.by_slot) for v in (on, low, high, dual)], 1).long(),
        # the factor, the coefficient, the sum and the product round once each
        grad=grad, e_grad=factor * (e_v + abs(kc) * (e_slope + U * slope.abs())) + 4 * U * factor * (
            v_slope.abs() + abs(kc) * slope.abs()) + 1e-38,
        grad_ent=-ec * factor, e_grad_ent=3 * U * abs(ec) * factor)


def _check_policy(plan, seed, options):
    torch = base._torch()
    rng = np.random.default_rng(seed)
    tiles = base._tiles(plan, plan.labels(rng, 0.4, 0.1), 1, 0, 0)
    maps = ref.Maps(plan, "cuda")
    gen = torch.Generator("cuda").manual_seed(seed)
    r = lambda n, sd=1.0: torch.randn(n, generator=gen, device="cuda") * sd
    lp = -r(plan.E, 2).abs()
    old, kref, ent = lp + r(plan.E, 0.25), lp + r(plan.E, 0.8), r(plan.E).abs() * 3
    advantages = r(plan.R), r(plan.E)
    w = torch.rand(plan.K, generator=gen, device="cuda", dtype=torch.float64)
    for kl, reduce, with_ent in options:
        token = (kl + reduce + with_ent) % 2
        p = base._policy_params(dict(kl=kl, reduce=reduce, token_advantage=token, kl_coef=0.3, entropy_coef=0.07 * with_ent,
                                     dual_clip=0.0 if kl == 2 else 1.4))
        log(f"policy {plan.E} elements: {p}")
        args = (lp, old, kref if kl else None, ent if with_ent else None, advantages[token], w)
        want = _policy64(maps, plan, tiles.labels, p, *args)
        out, status = base._policy_run(tiles, plan, p, *args, extra=0)
        assert int(status.item()) == 0
        assert torch.equal(out["counts"], want["counts"])
        for at in (1, 2) + ((3,) if p["dual_clip"] else ()):
            assert int(want["counts"][:, at].sum()) > 0
        for k in ("loss", "means", "grad") + (("grad_ent",) if with_ent else ()):
            err = (out[k].double() - want[k]).abs()
            assert torch.all(err <= want["e_" + k]), (p, k, float((err / want["e_" + k]).max()))
            if k.startswith("grad"):
                assert torch.all(out[k][~want["on"]] == 0)
        again, _ = base._policy_run(tiles, plan, p, *args, extra=0)
        for k, v in out.items():
            assert v is None or torch.equal(v, again[k]), k


EVERY = [(kl, reduce, ent) for kl in range(4) for reduce in range(3) for ent in (0, 1)]


def test_policy_in_one_block_by_option():
    plan = Plan([[70, 90, 81], [300], [], [33] * 30, [3] * 50, [700]], base=(3, 1 << 33))
    assert plan.E <= 4096
    _check_policy(plan, 3, EVERY)


def test_policy_passes_by_option():
    rng = np.random.default_rng(4)
    plan = Plan([sorted(int(v) for v in rng.integers(300, 500, 7)), [2000], [], [33] * 40, [3] * 300, [1] * 1500,
                 [1100, 1200], [14000]], base=(3, 1 << 33))
    assert plan.E > 4096
    _check_policy(plan, 5, EVERY)


@pytest.mark.parametrize("elems", [3_000_000, 6_000_000, 9_000_000, 18_000_000])
def test_policy_large_runs_by_option(elems):
    """Each size takes another length of chunk."""
    rng = np.random.default_rng(elems)
    groups, total = [], 0
    while total < elems:
        l = int(rng.choice([3, 40, 100, 256, 480, 1023, 4097])) + int(rng.integers(0, 3))
        n = max(1, int(rng.integers(2000, 60_000)) // l)
        groups += [[max(1, l - int(v)) for v in rng.integers(0, 1 + l // 9, n - 1)] + [l]]
        total += n * l
        if len(groups) % 9 == 0:
            groups.append([])
    _check_policy(Plan(groups, base=(11, 1 << 34)), elems, EVERY)
