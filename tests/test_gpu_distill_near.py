"""The distillation loss beside the teacher: a student that starts from its weights or has nearly learned it.  There
a divergence falls with the square of the distance and its slopes with the distance; both are compared relative to
themselves, with the definition in extended precision.

A probability costs up to 7 roundings, the series of a term or a logarithm and its products 11 more, a sum over a
list at most nine (three adds of a lane, six over the lanes): values and slopes are right to C = 40 roundings of
themselves where nothing but products stands between them and the inputs."""
import math

import numpy as np
import pytest

from _losses import U, Plan
from _parity import log
from test_gpu_distill import Run

pytestmark = pytest.mark.gpu

X = np.longdouble
C = 40
LISTED, RENORMALIZED, REST = 0, 1, 2
NOISE = [0.05, 1e-2, 1e-3, 1e-4]


def _near(rng, E, k, noise, mass=(0.6, 0.999)):
    """A teacher's lists and those of a student beside it: likeliest first, some lists end early."""
    z = -np.cumsum(rng.exponential(0.5, (E, k)), -1)
    t = z - np.log(np.exp(z).sum(-1, keepdims=True)) + np.log(rng.uniform(*mass, (E, 1)))
    s = t + noise * (rng.standard_normal((E, k)).clip(-4, 4) + rng.standard_normal((E, 1)).clip(-4, 4))
    t, s = t.astype(np.float32), s.astype(np.float32)
    none = np.arange(k)[None] >= np.where(rng.random(E) < 0.3, rng.integers(1, k + 1, E), k)[:, None]
    t[none] = -math.inf
    return t, s


def _extended(t, s):
    """Logs and probabilities of the entries, 0 for those that are none."""
    there = t != -math.inf
    t, s = np.where(there, t, 0).astype(X), np.where(there, s, 0).astype(X)
    return t, s, np.where(there, np.exp(t), 0), np.where(there, np.exp(s), 0), there


def _mixture(w, p, q, d):
    """Terms of the divergence from the mixture, and ln(q / m)."""
    w = X(w)
    less_p, less_q = -np.log1p((1 - w) * np.expm1(-d)), -np.log1p(w * np.expm1(d))
    return w * p * less_p + (1 - w) * q * less_q, less_q


def _run(t, s, kind, support, w):
    """Every token's value, in a slot of its own, and the slopes."""
    import paper_2606_19989_amd as odb
    E, k = t.shape
    params = odb.DistillParams(kind=kind, support=support, reduce=2, mix=w)
    y = np.zeros(E, np.int32)
    each, all_ = Run(Plan([[1]] * E), y, t, s, k, params, shift=0), Run(Plan([[1] * E]), y, t, s, k, params, shift=0)
    each()
    all_()
    value, slope = each.numpy()[1], each.numpy()[3]
    assert np.array_equal(slope, all_.numpy()[3])
    return value, slope


def _hold(name, got, want, tol):
    ratio = np.abs(got - want) / tol
    log(f"  {name}: {float(ratio.max()):.3f} of the tolerance")
    assert np.all(ratio <= 1), (name, float(ratio.max()))


@pytest.mark.parametrize("noise", NOISE)
@pytest.mark.parametrize("w", [0.3, 0.5, 1e-3, 0.999])
def test_mixture_of_listed_entries(w, noise):
    rng = np.random.default_rng(31)
    for E, k in ((700, 16), (200, 100), (900, 3)):
        log(f"distill near: mixture {w}, noise {noise}, k {k}")
        t, s = _near(rng, E, k, noise)
        value, grad = _run(t, s, 2, LISTED, w)
        t64, s64, p, q, _ = _extended(t, s)
        term, less_q = _mixture(w, p, q, t64 - s64)
        _hold("values", value, term.sum(-1), C * U * term.sum(-1) + 1e-37)
        assert np.all(value >= 0)
        slope = (1 - X(w)) * q * less_q
        _hold("slopes", grad, slope, C * U * np.abs(slope) + 2.0 ** -115)


@pytest.mark.parametrize("noise", [0.7, 3.0])
@pytest.mark.parametrize("w", [0.3, 1e-3, 0.999, 1e-6])
def test_mixture_of_a_small_weight(w, noise):
    """Away from the teacher a term is a sum of two of either sign, right to 100 roundings of those, and a logarithm
    to 100 of itself: one side's is taken, right to 3 of at most 16, and the distance leaves the other's, ln 2 or more."""
    rng = np.random.default_rng(32)
    t, s = _near(rng, 700, 16, noise)
    log(f"distill: mixture {w}, noise {noise}")
    value, grad = _run(t, s, 2, LISTED, w)
    t64, s64, p, q, _ = _extended(t, s)
    term, less_q = _mixture(w, p, q, t64 - s64)
    slope = (1 - X(w)) * q * less_q
    sizes = np.abs(slope) + np.abs(term - slope)
    _hold("values", value, term.sum(-1), 100 * U * sizes.sum(-1) + 1e-37)
    _hold("slopes", grad, slope, 100 * U * np.abs(slope) + 2.0 ** -115)


# Powers whose sums are taken from 1 are right to 2^-46.
WIDE = 2.0 ** -46


@pytest.mark.parametrize("mass", [(0.6, 0.999), (1 - 1e-3, 1 - 1e-5)])
@pytest.mark.parametrize("noise", NOISE)
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_with_the_rest(kind, noise, mass):
    """What the lists leave out is one entry more; its log's distance is right to a few roundings and to what the powers
    leave of it.  Where it is more than 1/2, or the rest is held, the rest's probabilities stand in its place."""
    w = 0.3
    rng = np.random.default_rng(33)
    for E, k in ((700, 16), (200, 100), (900, 3)):
        log(f"distill near: kind {kind} with the rest of {mass}, noise {noise}, k {k}")
        t, s = _near(rng, E, k, noise, mass)
        value, grad = _run(t, s, kind, REST, w)
        t64, s64, p, q, there = _extended(t, s)
        d = t64 - s64
        rp, rq = 1 - p.sum(-1), 1 - q.sum(-1)
        held = rq <= 2.0 ** -24
        rp, rq = np.maximum(rp, 2.0 ** -24), np.maximum(rq, 2.0 ** -24)
        x0, d0 = (rp - rq) / rq, np.log(rp) - np.log(rq)
        near = (np.abs(x0) < 0.49) & (np.abs(d0) < 0.49)
        assert near.any()
        if kind == 0:
            D = (p * d).sum(-1) + rp * d0
            slope = -p + q * np.where(held, 0, rp / rq)[:, None]
            size = np.where(near & ~held, p.T * np.abs(np.expm1(-d.T)) + q.T * np.abs(x0), p.T + q.T * rp / rq)
        elif kind == 1:
            D = -(q * d).sum(-1) - rq * d0
            slope = q * (np.where(held, 1, d0)[:, None] - d)
            size = q.T * (np.abs(d.T) + np.where(held, 1, np.abs(d0)))
        else:
            term, less_q = _mixture(w, p, q, d)
            term0, less_q0 = _mixture(w, rp, rq, d0)
            D = term.sum(-1) + term0
            slope = (1 - w) * q * (less_q - np.where(held, 0, less_q0)[:, None])
            size = (1 - w) * q.T * (np.abs(less_q.T) + np.abs(less_q0))
        wide = WIDE / np.minimum(rp, rq)
        # D is the sum of terms of none below 0 and of what the held rests add to the sums, `over`; that may be below 0
        # and leave less of D than the terms are, whose roundings count: they are D - over or D + over
        over = np.abs(p.sum(-1) + rp - q.sum(-1) - rq)
        tol = C * U * (np.abs(D) + 2 * over + np.where(near, 0, rp + rq)) + 4 * WIDE * np.abs(d0) + 1e-37
        _hold("values", value, D, tol)
        assert np.all(value[near & ~held] >= 0)
        tol = C * U * size.T + (4 * q * wide[:, None]) + 2.0 ** -115
        _hold("slopes", grad, np.where(there, slope, 0), tol)


@pytest.mark.parametrize("noise", NOISE)
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_renormalized(kind, noise):
    """Each side divided by its sum.  With G the largest distance of an entry's logs as they are, a distance less that of
    the sums' logs is right to d = 2 U G (S + 25): two roundings of G each for the entry's and the largest entries'
    distances, and powers whose exponents, S at most, are rounded, times distances of 2 G at most.  A value moves with
    the square of a distance that all entries are off by, and by 2 G U times the distances with each one's own."""
    w = 0.3
    rng = np.random.default_rng(34)
    for E, k in ((700, 16), (200, 100), (900, 3)):
        log(f"distill near: kind {kind} renormalised, noise {noise}, k {k}")
        t, s = _near(rng, E, k, noise)
        value, grad = _run(t, s, kind, RENORMALIZED, w)
        t64, s64, p, q, there = _extended(t, s)
        d = np.where(there, t64 - s64, 0)
        G = np.abs(d).max(-1, keepdims=True)
        S = np.where(there, np.maximum(t64.max(-1, keepdims=True, where=there, initial=-1e9) - t64,
                                       s64.max(-1, keepdims=True, where=there, initial=-1e9) - s64), 0).max(-1, keepdims=True)
        sp, sq = p.sum(-1, keepdims=True), q.sum(-1, keepdims=True)
        d, p, q = np.where(there, d - (np.log(sp) - np.log(sq)), 0), p / sp, q / sq
        assert np.abs(d).max() < 0.5
        off = 2 * U * G * (S + 25)
        if kind == 0:
            D, slope = (p * d).sum(-1), q - p
        elif kind == 1:
            D = -(q * d).sum(-1)
            slope = -q * (d + D[:, None])
        else:
            term, less_q = _mixture(w, p, q, d)
            D, slope = term.sum(-1), (1 - w) * q * (less_q - (q * less_q).sum(-1, keepdims=True))
        both = p + q
        # a list of one entry has D = 0, of which the oracle's own roundings (2^-63 of logs below 8) leave something
        tol = U * ((C + S[:, 0]) * D + 8 * G[:, 0] * (both * np.abs(d)).sum(-1)) + off[:, 0] ** 2 + 2.0 ** -60
        _hold("values", value, D, tol)
        assert np.all(value >= 0)
        far = np.abs(d) + (q * np.abs(d)).sum(-1, keepdims=True)
        _hold("slopes", grad, slope, both * (2 * off + (C + S) * U * far) + 2.0 ** -115)


@pytest.mark.parametrize("low", [-60.0, -95.0, -200.0, -1000.0])
@pytest.mark.parametrize("support", [LISTED, RENORMALIZED, REST])
def test_an_entry_that_only_the_teacher_gives(support, low):
    """However little the teacher gives it: a forward divergence is infinite, the others and all slopes are not."""
    t = np.tile(np.float32([-0.7, low, -1.5, -math.inf]), (300, 1))
    s = np.tile(np.float32([-0.6, -math.inf, -1.75, -math.inf]), (300, 1))
    for kind in range(3):
        value, slope = _run(t, s, kind, support, 0.3)
        assert np.all(value == math.inf) if kind == 0 else np.all((value > 0) & (value < 2)) or support == LISTED
        assert np.all(np.isfinite(value)) or kind == 0
        assert np.all(np.isfinite(slope)) and np.all(slope[:, 3] == 0)


@pytest.mark.parametrize("support", [LISTED, RENORMALIZED, REST])
def test_a_student_that_is_the_teacher(support):
    """Distances of 0.  Renormalised lists' are off by e, 2 U at most (a reciprocal's and a product's rounding), which the
    slopes have taken off to 8 U e."""
    rng = np.random.default_rng(35)
    for E, k in ((500, 16), (100, 128), (300, 1)):
        t, _ = _near(rng, E, k, 0.1)
        s = np.where(t == -math.inf, 3.0, t).astype(np.float32)
        for kind in range(3):
            value, slope = _run(t, s, kind, support, 0.3)
            assert np.all((value >= 0) & (value <= U * U)), (kind, k)
            if support == LISTED and kind < 2:
                p = np.where(t == -math.inf, 0, np.exp(t.astype(X)))
                assert np.all(np.abs(slope - (p if kind else -p)) <= 4 * U * p + 2.0 ** -115)
            else:
                assert np.all(np.abs(slope) <= 16 * U * U), (kind, k)
