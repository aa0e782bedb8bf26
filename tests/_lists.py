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
