"""The operators over lists of tokens in 64 bits on the CPU, token by token from their definitions (numpy)."""
import math

import numpy as np

from _losses import IGNORE, U


def counted(labels, rows, cols, V, shift):
    """Which tokens of a tile count."""
    on = np.ones((rows, cols), bool) if labels is None else (labels >= 0) & (labels < V)
    on[:, :shift] = False
    return on


def _softmax(row, scale):
    m = row.max()
    x = scale * (row - m)
    e = np.exp(x)
    return m, x, e, e.sum()


def list_logprobs(z, labels, ids, shift, scale):
    """z [rows, cols, V] float64, ids [rows, cols, k]: list log-probabilities, stats."""
    rows, cols, V = z.shape
    out, stats = np.zeros(ids.shape), np.zeros((rows, cols, 2))
    for i, c in zip(*np.nonzero(counted(labels, rows, cols, V, shift))):
        m, x, e, s = _softmax(z[i, c - shift], scale)
        stats[i, c] = m, math.log(s)
        for j, v in enumerate(ids[i, c]):
            if 0 <= v < V:
                out[i, c, j] = x[v] - math.log(s)
    return out, stats


def list_logprobs_grad(z, labels, ids, shift, scale, g):
    """Gradient by z (float64) of sum g * list_logprobs."""
    rows, cols, V = z.shape
    out = np.zeros_like(z)
    for i, c in zip(*np.nonzero(counted(labels, rows, cols, V, shift))):
        real = (ids[i, c] >= 0) & (ids[i, c] < V)
        if not np.any(g[i, c][real] != 0):
            continue
        _, _, e, s = _softmax(z[i, c - shift], scale)
        d = -g[i, c][real].sum() * e / s
        np.add.at(d, ids[i, c][real], g[i, c][real])
        out[i, c - shift] = scale * d
    return out


def top(row, k):
    """The k largest entries above -inf of a row: of equal ones the first."""
    order = np.argsort(-row, kind="stable")[:k]
    return order[row[order] > -math.inf]


def rank(row, y):
    return int(np.sum((row > row[y]) | ((row == row[y]) & (np.arange(row.size) < y))))


def sum_bounds(V, bytes_each, x2, L):
    """Absolute error of a position's logsum: a thread adds at most V / G terms and ten levels are joined; every
    term's exponent and power and every rescaling add (3 |x| + 3) U, and sum p |x| <= sqrt(sum p x^2) = x2."""
    row = V * bytes_each
    G = 8 if row <= 1024 else 32 if row <= 2048 else 64 if row <= 16384 else 256
    return U * (V / G + 48 + 3 * x2 + 2 * np.abs(L))


def spread(row, scale):
    """sqrt(sum p x^2), x = scale * (row - largest)."""
    _, x, e, s = _softmax(row, scale)
    p = e / s
    return math.sqrt(np.sum(np.where(p > 0, p * np.where(p > 0, x, 0.0) ** 2, 0.0)))


# ------------------------------------------------------------------ distillation
LISTED, RENORMALIZED, REST = 0, 1, 2
LEAST = 2.0 ** -24


def _terms(kind, w, p, q, t, s):
    """Terms of a divergence between probabilities (with their logs) and their slopes by the student's log."""
    with np.errstate(all="ignore"):
        if kind == 0:
            return np.where(p > 0, p * (t - s), 0.0), -p
        if kind == 1:
            return np.where(q > 0, q * (s - t), 0.0), np.where(q > 0, q * (s - t + 1), 0.0)
        d = t - s
        less_p = np.where(d < -30, d - np.log(w * np.exp(d) + 1 - w), -np.log1p((1 - w) * np.expm1(np.minimum(-d, 30))))
        less_q = np.where(d > 30, -d - np.log(w + (1 - w) * np.exp(-d)), -np.log1p(w * np.expm1(np.minimum(d, 30))))
        slope = np.where(q > 0, (1 - w) * q * less_q, 0.0)
        return np.where(p > 0, w * p * less_p, 0.0) + slope, slope


def distill_token(t, s, kind, support, w):
    """(value, slopes [k], bound of the value's error, bounds of the slopes' errors), the bounds in units of U.

    A probability's exponent has an error of (|t| + |s| + what normalises them) U and its power a few more, a
    term and a slope as much times their sizes; a logarithm of a mixture as much over its smaller weight."""
    there = t != -math.inf
    slopes, e_slope = np.zeros(t.size), np.zeros(t.size)
    if support != REST and not there.any():
        return 0.0, slopes, 0.0, e_slope
    t0, s0 = t[there], s[there]
    size = np.abs(t0) + np.abs(np.where(np.isfinite(s0), s0, 0.0)) + 4.0
    if support == RENORMALIZED:
        lt, ls = (v.max() + math.log(np.exp(v - v.max()).sum()) for v in (t0, s0))
        size = size + abs(lt) + abs(ls) + 2 * (np.abs(t0 - t0.max()) + np.abs(np.where(np.isfinite(s0), s0 - s0.max(), 0.0)))
        t0, s0 = t0 - lt, s0 - ls
    p, q = np.exp(t0), np.exp(s0)
    term, slope = _terms(kind, w, p, q, t0, s0)
    value = term.sum()
    d = np.where(np.isfinite(s0), np.abs(t0 - s0), 0.0)
    c = 1.0 if kind != 2 else 1.0 / min(w, 1 - w)
    each = 4 * c * size * ((p if kind != 1 else 0) * (1 + d) + (q if kind != 0 else 0) * (1 + d))
    e_value, e = each.sum() + 12 * np.abs(np.where(np.isfinite(term), term, 0.0)).sum(), each.copy()
    if support == RENORMALIZED:
        total = slope.sum()
        slope = slope - q * total
        e = e + q * (each.sum() + 12 * np.abs(term).sum() + 4 * size * (1 + np.abs(total)))
    elif support == REST:
        rp, rq = 1 - p.sum(), 1 - q.sum()
        held = rq <= LEAST
        rp, rq = max(rp, LEAST), max(rq, LEAST)
        a, b = _terms(kind, w, np.array([rp]), np.array([rq]), np.log([rp]), np.log([rq]))
        value += a[0]
        moves = 0.0 if held else b[0] / rq
        slope = slope - q * moves
        e = e + 4 * q * (size * (1 + abs(moves)))
    slopes[there], e_slope[there] = slope, e
    return value, slopes, e_value, e_slope


def distill(plan, labels, student, teacher, k, kind, support, reduce, w, slot_weight, loss_scale, shift):
    """Losses, means and counts per slot, gradients [E, k], and bounds of the errors of means and gradients (U)."""
    K, E = plan.K, plan.E
    on = plan.counted(labels, shift)
    slot = plan.slot_of_row[plan.row_of]
    count = np.bincount(slot[on], minlength=K).astype(np.int64)
    per_row = np.bincount(plan.row_of[on], minlength=plan.R)
    rows = np.bincount(plan.slot_of_row[per_row > 0], minlength=K)
    mean, grad = np.zeros(K), np.zeros((E, k))
    e_mean, e_grad = np.zeros(K), np.zeros((E, k))
    for e in np.nonzero(on)[0]:
        r, j = plan.row_of[e], slot[e]
        f = 1.0 if reduce == 2 else 1.0 / count[j] if reduce == 0 else 1.0 / (per_row[r] * rows[j])
        v, g, ev, eg = distill_token(teacher[e], student[e], kind, support, w)
        sw = 1.0 if slot_weight is None else slot_weight[j]
        mean[j] += f * v
        grad[e] = loss_scale * sw * f * g
        e_mean[j] += f * ev
        e_grad[e] = abs(loss_scale * sw * f) * eg
    loss = loss_scale * (1.0 if slot_weight is None else slot_weight) * mean
    return loss, mean, count, grad, e_mean, e_grad
