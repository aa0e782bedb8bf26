"""The loss operators in 64 bits on the CPU, token by token from their definitions (numpy), and
tiles to run them on."""
import math

import numpy as np

IGNORE = -100
U = 2.0 ** -24          # half a step of fp32, relative


def token_logprobs(z, labels, shift, scale):
    """z [rows, cols, V] float64, labels [rows, cols]: logprob, stats, entropy, all [rows, cols]
    (stats with 2), and the per-token magnitudes that bound rounding errors."""
    rows, cols, V = z.shape
    lp, stats, ent = np.zeros((rows, cols)), np.zeros((rows, cols, 2)), np.zeros((rows, cols))
    second = np.zeros((rows, cols))       # sum p x^2, x = scale * (z - largest)
    at = np.zeros((rows, cols))           # |x| of the label
    for i in range(rows):
        for c in range(shift, cols):
            y = labels[i, c]
            if y == IGNORE or y < 0 or y >= V:
                continue
            row = z[i, c - shift]
            m = row.max()
            x = scale * (row - m)
            e = np.exp(x)
            s = e.sum()
            lp[i, c] = x[y] - math.log(s)
            stats[i, c] = m, math.log(s)
            p = e / s
            ex = np.where(p > 0, p * np.where(p > 0, x, 0.0), 0.0)
            ent[i, c] = math.log(s) - ex.sum()
            second[i, c] = np.where(p > 0, p * np.where(p > 0, x, 0.0) ** 2, 0.0).sum()
            at[i, c] = abs(x[y])
    return lp, stats, ent, second, at


def token_logprobs_grad(z, labels, shift, scale, g, h):
    """Gradient with respect to z (float64); g, h [rows, cols] (h may be None)."""
    rows, cols, V = z.shape
    out = np.zeros_like(z)
    for i in range(rows):
        for c in range(shift, cols):
            y = labels[i, c]
            if y == IGNORE or y < 0 or y >= V:
                continue
            hc = 0.0 if h is None else h[i, c]
            if g[i, c] == 0 and hc == 0:
                continue
            row = z[i, c - shift]
            x = scale * (row - row.max())
            lse = math.log(np.exp(x).sum())
            lnp = x - lse
            p = np.exp(lnp)
            d = -g[i, c] * p
            d[y] += g[i, c]
            if hc:
                H = -np.where(p > 0, p * np.where(p > 0, lnp, 0.0), 0.0).sum()
                d -= hc * np.where(p > 0, p * (np.where(p > 0, lnp, 0.0) + H), 0.0)
            out[i, c - shift] = scale * d
    return out


class Plan:
    """Slot arrays over rows of given lengths: groups is a list of lists of row lengths, one a
    slot ([] is an IDLE slot).  `base` puts other slots in front (offsets that do not start at 0)."""

    def __init__(self, groups, base=(0, 0)):
        self.rows = np.array([len(g) for g in groups], np.int32)
        self.maxlen = np.array([max(g) if g else 0 for g in groups], np.int32)
        self.row_off = base[0] + np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int64)
        self.tile_off = base[1] + np.concatenate([[0], np.cumsum(self.rows.astype(np.int64) * self.maxlen)]).astype(np.int64)
        self.K, self.R = len(groups), int(self.rows.sum())
        self.E = int(self.tile_off[-1] - self.tile_off[0])
        row_max = np.repeat(self.maxlen.astype(np.int64), self.rows)
        start = np.cumsum(row_max) - row_max
        self.row_of = np.repeat(np.arange(self.R), row_max)
        self.col_of = np.arange(self.E) - start[self.row_of]
        self.slot_of_row = np.repeat(np.arange(self.K), self.rows)
        self.lens = np.array([l for g in groups for l in g], np.int64)

    def labels(self, rng, prompt=0.0, empty=0.0, vocab=100):
        y = rng.integers(0, vocab, self.E).astype(np.int32)
        real = self.col_of < self.lens[self.row_of]
        if prompt:
            first = (rng.random(self.R) * prompt * self.lens).astype(np.int64)
            first = np.where(rng.random(self.R) < empty, self.lens, first)
            real &= self.col_of >= first[self.row_of]
        y[~real] = IGNORE
        return y

    def counted(self, labels, shift):
        return (labels != IGNORE) & (self.col_of >= shift)


def kl_term(mode, x):
    if mode == 0:
        return 0.0, 0.0
    if mode == 1:
        return x, 1.0
    if mode == 2:
        return 0.5 * x * x, x
    return math.expm1(-x) + x, -math.expm1(-x)


def policy_token(lp, old, ref, adv, p):
    """(policy, KL, ratio, d policy, d KL, clip kind) of one token; p: dict of parameters."""
    d = lp - old
    try:
        r = math.exp(d)
    except OverflowError:
        r = math.inf
    low = math.log1p(-p["clip_low"]) if p["clip_low"] < 1 else -math.inf
    high = math.log1p(p["clip_high"])
    dual = math.log(p["dual_clip"]) if p["dual_clip"] else math.inf
    kl, dkl = kl_term(p["kl"], lp - ref)
    if adv == 0:
        return 0.0, kl, r, 0.0, dkl, 0
    if adv > 0 and d > high:
        return -(1 + p["clip_high"]) * adv, kl, r, 0.0, dkl, 2
    if adv < 0 and d < low:
        return -(1 - p["clip_low"]) * adv, kl, r, 0.0, dkl, 1
    if adv < 0 and d > dual:
        return -p["dual_clip"] * adv, kl, r, 0.0, dkl, 3
    return -r * adv, kl, r, -r * adv, dkl, 0


def policy_loss(plan, labels, shift, p, lp, old, ref, ent, adv, weight):
    """Everything odb_policy_loss writes, and the sums of magnitudes that bound its rounding."""
    on = plan.counted(labels, shift)
    K = plan.K
    slot = plan.slot_of_row[plan.row_of]
    n_slot = np.bincount(slot[on], minlength=K)
    n_row = np.bincount(plan.row_of[on], minlength=plan.R)
    n_rows = np.bincount(plan.slot_of_row[n_row > 0], minlength=K)
    loss, means, mags = np.zeros(K), np.zeros((K, 4)), np.zeros((K, 4))
    counts = np.zeros((K, 4), np.int64)
    counts[:, 0] = n_slot
    grad, grad_mag, grad_ent = np.zeros(plan.E), np.zeros(plan.E), np.zeros(plan.E)
    for e in np.nonzero(on)[0]:
        k, row = slot[e], plan.row_of[e]
        w = [1.0 / n_slot[k], 1.0 / (float(n_row[row]) * n_rows[k]), 1.0][p["reduce"]]
        a = float(adv[e] if p["token_advantage"] else adv[row])
        l = float(lp[e])
        v = policy_token(l, l if old is None else float(old[e]), 0.0 if ref is None else float(ref[e]), a, p)
        h = 0.0 if ent is None else float(ent[e])
        terms = np.array([v[0], v[1], h, v[2]])
        means[k] += w * terms
        mags[k] += w * np.abs(terms)
        if v[5]:
            counts[k, v[5]] += 1
        scale = p["loss_scale"] * (1.0 if weight is None else float(weight[k]))
        grad[e] = scale * w * (v[3] + p["kl_coef"] * v[4])
        grad_mag[e] = abs(scale * w) * (abs(v[3]) + abs(p["kl_coef"]) * max(abs(v[4]), abs(l) if ref is None else
                                                                             abs(l - float(ref[e]))))
        grad_ent[e] = -p["entropy_coef"] * scale * w
    for k in range(K):
        if n_slot[k]:
            loss[k] = p["loss_scale"] * (1.0 if weight is None else float(weight[k])) * (
                means[k, 0] + p["kl_coef"] * means[k, 1] - p["entropy_coef"] * means[k, 2])
    return dict(loss=loss, means=means, counts=counts, grad=grad, grad_ent=grad_ent, mags=mags, grad_mag=grad_mag)


def preference_loss(plan, labels, shift, p, lp, ref, row_ids, pair):
    on = plan.counted(labels, shift)
    x = np.where(on, lp.astype(np.float64), 0.0)
    if ref is not None:
        x = x - np.where(on, ref.astype(np.float64), 0.0)
    R = plan.R
    S = np.array([math.fsum(x[(plan.row_of == r) & on]) for r in range(R)])
    n = np.bincount(plan.row_of[on], minlength=R)
    per = 1.0 / np.maximum(n, 1) if p["normalize"] else np.ones(R)
    S = S * per
    row_of = {}
    for r in range(R):
        row_of.setdefault(r if row_ids is None else int(row_ids[r]), r)
    row_loss, coef = np.zeros(R), np.zeros(R)
    pairs = right = 0
    for a, r in row_of.items():
        v = int(pair[a])
        if v <= 0:
            continue
        q = row_of.get(v - 1)
        if q is None:
            continue
        h = p["beta"] * (S[r] - S[q]) - p["margin"]
        if p["kind"] == 0:
            e = p["label_smoothing"]
            L = (1 - e) * np.logaddexp(0, -h) + e * np.logaddexp(0, h)
            sig = lambda t: 1 / (1 + math.exp(-t)) if t > -700 else 0.0
            dh = e * sig(h) - (1 - e) * sig(-h)
        elif p["kind"] == 1:
            L, dh = max(0.0, 1 - h), -1.0 if h < 1 else 0.0
        else:
            L, dh = ((h - 0.5) / p["beta"]) ** 2, 2 * (h - 0.5) / p["beta"] ** 2
        row_loss[r] = p["loss_scale"] * L
        coef[r] += p["loss_scale"] * p["beta"] * dh * per[r]
        coef[q] -= p["loss_scale"] * p["beta"] * dh * per[q]
        pairs += 1
        right += S[r] > S[q]
    return dict(loss=math.fsum(row_loss), row_loss=row_loss, reward=p["beta"] * S, counts=np.array([pairs, right]),
                grad=np.where(on, coef[plan.row_of], 0.0))


# ------------------------------------------------------------------ large runs, on the GPU in 64 bits
class Maps:
    """Row, column and slot of every element, and sums over a row's or a slot's elements."""

    def __init__(self, plan, device):
        import torch
        rows, maxlen = torch.from_numpy(plan.rows).long().to(device), torch.from_numpy(plan.maxlen).long().to(device)
        self.by_row = torch.repeat_interleave(maxlen, rows)
        self.by_slot, self.rows_of_slot = rows * maxlen, rows
        start = torch.cumsum(self.by_row, 0) - self.by_row
        self.row = torch.repeat_interleave(torch.arange(plan.R, device=device), self.by_row)
        self.slot = torch.repeat_interleave(torch.arange(plan.K, device=device), rows)[self.row]
        self.col = torch.arange(plan.E, device=device) - start[self.row]

    @staticmethod
    def sum(v, lengths):
        import torch
        return torch.segment_reduce(v.double(), "sum", lengths=lengths, initial=0.0, unsafe=True)


def policy_loss_torch(m, labels, shift, p, lp, old, ref, adv):
    """Loss, means, counts and gradient (kl 3, an advantage per row, no slot weights)."""
    import torch
    on = (labels != IGNORE) & (m.col >= shift)
    n_slot, n_row = m.sum(on, m.by_slot), m.sum(on, m.by_row)
    n_rows = m.sum(n_row > 0, m.rows_of_slot)
    zero = torch.zeros((), dtype=torch.float64, device=on.device)
    w = [lambda: 1 / n_slot[m.slot], lambda: 1 / (n_row[m.row] * n_rows[m.slot]), lambda: zero + 1][p["reduce"]]()
    w = torch.where(on, w, zero)
    d, A, x = lp.double() - old.double(), adv[m.row].double(), lp.double() - ref.double()
    r = d.exp()
    low = on & (A < 0) & (d < math.log1p(-p["clip_low"]))
    high = on & (A > 0) & (d > math.log1p(p["clip_high"]))
    pol = -torch.where(high, 1 + p["clip_high"], torch.where(low, 1 - p["clip_low"], r)) * A
    kl = torch.expm1(-x) + x
    means = [m.sum(w * v, m.by_slot) for v in (pol, kl, r * 0, r)]
    mags = [m.sum(w * v.abs(), m.by_slot) for v in (pol, kl, r * 0, r)]
    slope = torch.where(low | high, zero, pol)
    counts = torch.stack([n_slot, m.sum(low, m.by_slot), m.sum(high, m.by_slot), n_slot * 0], 1).long()
    s = p["loss_scale"]
    return dict(loss=s * (means[0] + p["kl_coef"] * means[1]), means=torch.stack(means, 1), mags=torch.stack(mags, 1),
                counts=counts, grad=s * w * (slope - p["kl_coef"] * torch.expm1(-x)),
                grad_mag=s * w * (slope.abs() + p["kl_coef"] * torch.maximum(x.abs(), torch.expm1(-x).abs())))


def preference_loss_torch(m, labels, shift, p, lp, ref, row_ids, pair):
    """Loss, rows' losses and rewards, counts and gradient of the sigmoid; every id has one row."""
    import torch
    on = (labels != IGNORE) & (m.col >= shift)
    zero = torch.zeros((), dtype=torch.float64, device=on.device)
    S = m.sum(torch.where(on, lp.double() - ref.double(), zero), m.by_row)
    n = m.sum(on, m.by_row).clamp(min=1) if p["normalize"] else torch.ones_like(S)
    S = S / n
    row_of = torch.empty_like(row_ids).long()
    row_of[row_ids.long()] = torch.arange(row_ids.numel(), device=on.device)
    a = torch.nonzero(pair > 0)[:, 0]
    c, r = row_of[a], row_of[pair[a].long() - 1]
    h = p["beta"] * (S[c] - S[r])
    loss, coef = torch.zeros_like(S), torch.zeros_like(S)
    loss[c] = p["loss_scale"] * torch.nn.functional.softplus(-h)
    coef[c] = -p["loss_scale"] * p["beta"] * torch.sigmoid(-h)
    coef[r] = -coef[c]
    coef = coef / n
    return dict(loss=loss.sum(), row_loss=loss, reward=p["beta"] * S, grad=torch.where(on, coef[m.row], zero),
                counts=torch.stack([torch.tensor(a.numel(), device=on.device), (S[c] > S[r]).sum()]))
