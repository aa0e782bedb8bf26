"""The loss operators whose speed counts: from the logits of a collated tile to a weighted loss
and its gradient.

A trainer runs its model on the tiles that the plan collates, takes the log-probabilities of the
labels from the logits (:func:`odb_token_logprobs`), turns them into a clipped policy loss with a
KL term (:func:`odb_policy_loss`) or a preference loss over pairs of rows
(:func:`odb_preference_loss`), both with their gradient, and hands that back to the logits
(:func:`odb_token_logprobs_backward`).  The cases are those calls from one token to whole windows
of tiles: prompts and padding that do not count, rows in which nothing counts, vocabularies that
are odd or end in masked columns, logits with strides, every type and option.

``run`` computes an operator in its plain form (elementary torch operations, fp32 rounded once at
the end; fp64 for long sums and for values next to a border) or, with ``own``, through the
framework's entry points.
"""
import math

import numpy as np
import torch

own = False

IGNORE = -100
_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
KL = {"none": 0, "linear": 1, "square": 2, "exp": 3}
REDUCE = {"token_mean": 0, "row_mean": 1, "sum": 2}
PREFERENCE = {"sigmoid": 0, "hinge": 1, "square": 2}


def listed():
    return [
        # the score of one next token, as a server asks for it: the cost of a launch
        {"name": "logprobs_one", "kind": "logprobs", "rows": 1, "cols": 1, "vocab": 32000, "dtype": "bf16", "shift": 0},
        # a small ragged tile behind a model that answers in fp32, prompts masked, an odd vocabulary with a
        # padded stride and masked columns, temperature and entropy
        {"name": "logprobs_ragged", "kind": "logprobs", "rows": 7, "cols": 301, "vocab": 50021, "dtype": "fp32",
         "shift": 1, "prompt": 0.3, "pad": 11, "masked_columns": 21, "scale": 1.25, "entropy": True},
        # half a 16,384-token tile at the benchmark's vocabulary: the log-probabilities of a training step
        {"name": "logprobs_tile", "kind": "logprobs", "rows": 16, "cols": 512, "vocab": 151936, "dtype": "bf16",
         "shift": 1},
        # the gradient of a few short rows over a small vocabulary, with an entropy bonus
        {"name": "grad_small", "kind": "grad", "rows": 3, "cols": 17, "vocab": 1000, "dtype": "fp16", "shift": 1,
         "scale": 0.8, "entropy": True},
        # an ordinary step's: an odd vocabulary, prompts masked, a fifth of the tokens clipped (no gradient)
        {"name": "grad_ordinary", "kind": "grad", "rows": 5, "cols": 509, "vocab": 65537, "dtype": "bf16", "shift": 1,
         "prompt": 0.25, "zeros": 0.2},
        # the gradient of a whole training step at the benchmark's vocabulary
        {"name": "grad_tile", "kind": "grad", "rows": 8, "cols": 512, "vocab": 151936, "dtype": "bf16", "shift": 1},
        # a handful of short answers: the cost of the launches
        {"name": "policy_small", "kind": "policy", "elems": 256, "mean_len": 40, "budget": 0, "kl": "exp",
         "reduce": "token_mean"},
        # one rank's step: a 16,384-token tile, the mean of row means, an entropy bonus, prompts masked
        {"name": "policy_step", "kind": "policy", "elems": 16384, "mean_len": 480, "budget": 0, "kl": "exp",
         "reduce": "row_mean", "entropy": True, "prompt": True},
        # the tiles of a whole window at once, each with its loss-scaling weight
        {"name": "policy_window", "kind": "policy", "elems": 1 << 26, "mean_len": 480, "budget": 32768, "kl": "exp",
         "reduce": "token_mean", "prompt": True, "dual_clip": 3.0},
        # one rank's step of pairs by row number
        {"name": "preference_step", "kind": "preference", "elems": 16384, "mean_len": 480, "budget": 0,
         "loss": "sigmoid", "prompt": True},
        # a small window of ragged rows, pairs by sample id spread over its tiles, averaged per row, no reference
        {"name": "preference_ragged", "kind": "preference", "elems": 1 << 20, "mean_len": 170, "budget": 8192,
         "loss": "sigmoid", "ids": True, "normalize": True, "reference": False, "margin": 0.5},
        # the tiles of a whole window, pairs by sample id
        {"name": "preference_window", "kind": "preference", "elems": 1 << 26, "mean_len": 480, "budget": 32768,
         "loss": "sigmoid", "ids": True, "prompt": True, "smoothing": 0.1},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["logprobs", "grad", "policy", "preference"])
    c = {"kind": kind}
    if kind in ("logprobs", "grad"):
        c["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        c["vocab"] = log(33, 200000)
        most = (1 << 30) // _BYTES[c["dtype"]] // c["vocab"]          # at most 1 GiB of logits
        tokens = log(1, max(2, min(65536, most)))
        c["rows"] = min(tokens, log(1, 64))
        c["cols"] = max(1, tokens // c["rows"])
        c["shift"] = rng.choice([0, 1, 1])
        if rng.random() < 0.5:
            c["prompt"] = round(rng.uniform(0.05, 0.6), 3)
        if rng.random() < 0.4:
            c["pad"] = rng.randrange(1, 70)
        if rng.random() < 0.3:
            c["masked_columns"] = rng.randrange(1, max(2, c["vocab"] // 4))
        if rng.random() < 0.4:
            c["scale"] = round(rng.uniform(0.5, 2.0), 3)
        c["entropy"] = rng.random() < 0.4
        if kind == "grad" and rng.random() < 0.5:
            c["zeros"] = round(rng.uniform(0.05, 0.5), 3)
        if not _counted_rows(c).sum():      # a single token is scored by its own logits
            c["shift"] = 0
        return c
    c["mean_len"] = log(5, 2000)
    c["elems"] = log(100, 1 << 25)
    one = rng.random() < 0.4
    if one:
        c["elems"] = min(c["elems"], 1 << 17)
    c["budget"] = 0 if one else log(2048, 131072)
    c["prompt"] = rng.random() < 0.6
    if kind == "policy":
        c["kl"] = rng.choice(list(KL))
        c["reduce"] = rng.choice(list(REDUCE))
        c["entropy"] = rng.random() < 0.3
        c["token_advantage"] = rng.random() < 0.3
        c["old"] = rng.random() < 0.85
        if rng.random() < 0.3:
            c["dual_clip"] = round(rng.uniform(1.5, 5.0), 2)
    else:
        c["loss"] = rng.choice(list(PREFERENCE))
        c["ids"] = rng.random() < 0.6
        c["normalize"] = rng.random() < 0.3
        c["reference"] = rng.random() < 0.7
        c["margin"] = round(rng.uniform(0.0, 1.0), 2) if rng.random() < 0.4 else 0.0
        c["smoothing"] = round(rng.uniform(0.0, 0.3), 2) if c["loss"] == "sigmoid" and rng.random() < 0.4 else 0.0
    return c


# ------------------------------------------------------------------------------ inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _row_lengths(case):
    """Real tokens of every row of a tile: up to a tenth shorter than the longest."""
    i, cols = np.arange(case["rows"], dtype=np.int64), case["cols"]
    return cols - (i * 7919) % (cols // 10 + 1)


def _counted_rows(case):
    """Scored tokens of every row of a tile (work without inputs)."""
    lens = _row_lengths(case)
    first = np.maximum((case.get("prompt", 0.0) * lens).astype(np.int64), case["shift"])
    return np.maximum(lens - first, 0)


def _logits_case(case, seed):
    dev = _device()
    gen = torch.Generator(dev).manual_seed(seed)
    rows, cols, V = case["rows"], case["cols"], case["vocab"]
    dtype = _DTYPES[case["dtype"]]
    lens = torch.from_numpy(_row_lengths(case)).to(dev)
    c = torch.arange(cols, device=dev)
    first = (case.get("prompt", 0.0) * lens.double()).long()
    real = (c[None, :] >= first[:, None]) & (c[None, :] < lens[:, None])
    usable = V - min(case.get("masked_columns", 0), V - 1)
    labels = torch.randint(0, usable, (rows, cols), generator=gen, device=dev, dtype=torch.int32)
    labels = torch.where(real, labels, torch.full_like(labels, IGNORE))
    # a model's logits: noise, the label ahead of it by a varying lead; columns beyond the vocabulary masked
    wide = torch.empty(rows, cols, V + case.get("pad", 0), dtype=dtype, device=dev)
    for r in range(rows):
        wide[r].copy_(torch.randn(wide[r].shape, generator=gen, device=dev, dtype=torch.float32) * 2.5)
    logits = wide[:, :, :V]
    sh = case["shift"]
    rr, cc = torch.nonzero((labels != IGNORE) & (c[None, :] >= sh), as_tuple=True)
    y = labels[rr, cc].long()
    lead = torch.rand(rr.numel(), generator=gen, device=dev) * 14.0
    logits[rr, cc - sh, y] = lead.to(dtype)
    if usable < V:
        logits[:, :, usable:] = -math.inf if V % 2 else torch.finfo(dtype).min
    return logits, labels, rr, cc, y, gen


def _lengths(case):
    """Realised lengths of the rows of a policy or preference case, about case["elems"] tokens: the
    same ones in every window, so that its arrays keep their sizes; whose they are differs."""
    rng = np.random.default_rng(480)
    mean = min(case["mean_len"], max(1, case["elems"] // 2))
    n = max(2, case["elems"] // mean)
    s2 = math.log1p(0.8 ** 2)
    l = np.exp(math.log(mean) - s2 / 2 + math.sqrt(s2) * rng.standard_normal(n))
    if case["budget"] == 0:    # one tile: rows of like length, as grouping makes them
        l = mean * (0.85 + 0.15 * rng.random(n))
    return np.clip(np.round(l), 1, 16384).astype(np.int64)


def _tiles(case, seed):
    """Slot arrays of a plan, row ids, labels and the element -> row and column maps."""
    dev = _device()
    rng = np.random.default_rng(seed)
    gen = torch.Generator(dev).manual_seed(seed)
    lens = rng.permutation(_lengths(case))
    n = len(lens)
    order = np.argsort(-lens, kind="stable")
    rows, maxlen, ids = [], [], []
    a = 0
    while a < n:
        b = n if case["budget"] == 0 else min(n, a + max(case["budget"] // int(lens[order[a]]), 1))
        rows.append(b - a)
        maxlen.append(int(lens[order[a]]))
        ids.append(order[a:b][::-1])           # a tile's rows run short to long
        a = b
    if case["budget"]:                         # some ranks have no tile at the last step
        rows += [0, 0]
        maxlen += [0, 0]
    ids = np.concatenate(ids)
    rows, maxlen = np.array(rows), np.array(maxlen)
    row_off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)
    tile_off = np.concatenate([[0], np.cumsum(rows * maxlen)]).astype(np.int64)
    dv = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(device=dev, dtype=t)
    s = {"slot_rows": dv(rows, torch.int32), "slot_maxlen": dv(maxlen, torch.int32),
         "slot_row_off": dv(row_off, torch.int64), "slot_tile_off": dv(tile_off, torch.int64),
         "row_ids": dv(ids, torch.int32), "num_rows": n, "num_elems": int(tile_off[-1])}
    row, col = _maps(s)
    row_len = dv(lens[ids], torch.int64)
    first = torch.zeros(n, dtype=torch.int64, device=dev)
    if case.get("prompt"):
        u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
        first = (u * 0.7 * row_len).long()
        first = torch.where(torch.rand(n, generator=gen, device=dev) < 0.02, row_len, first)   # nothing to learn
    real = (col >= first[row]) & (col < row_len[row])
    labels = torch.randint(0, 32000, (s["num_elems"],), generator=gen, device=dev, dtype=torch.int32)
    s["labels"] = torch.where(real, labels, torch.full_like(labels, IGNORE))
    return s, real & (col >= 1), gen


def _logprobs_like(counted, gen):
    """Log-probabilities as a model gives them: most near 0, some far below; 0 where nothing counts."""
    x = torch.randn(counted.numel(), generator=gen, device=counted.device)
    x = -(x * x * x * x).clamp(max=16.0)
    return torch.where(counted, x, torch.zeros_like(x))


def prepare(case, seed):
    kind = case["kind"]
    state = {"case": case}
    if kind in ("logprobs", "grad"):
        logits, labels, rr, cc, y, gen = _logits_case(case, seed)
        rows, cols, V = logits.shape
        dev, sh = logits.device, case["shift"]
        state.update(logits=logits, labels=labels, scale=float(case.get("scale", 1.0)))
        f32 = dict(dtype=torch.float32, device=dev)
        if kind == "grad":     # what the forward call left: (largest, log of the sum) and entropy of each token
            stats, ent = torch.zeros(rows, cols, 2, **f32), torch.zeros(rows, cols, **f32)
            for a, b in _blocks(rr.numel(), V):
                z = logits[rr[a:b], cc[a:b] - sh].double()
                m = z.amax(-1, keepdim=True)
                x = state["scale"] * (z - m)
                e = x.exp()
                t = e.sum(-1, keepdim=True)
                stats[rr[a:b], cc[a:b]] = torch.cat([m, t.log()], -1).float()
                ent[rr[a:b], cc[a:b]] = (t.log() - (e * x.clamp(min=-1e4)).sum(-1, keepdim=True) / t).float()[:, 0]
            g = torch.zeros(rows, cols, **f32)
            v = torch.randn(rr.numel(), generator=gen, **f32)
            if case.get("zeros"):
                v = torch.where(torch.rand(rr.numel(), generator=gen, device=dev) < case["zeros"],
                                torch.zeros_like(v), v)
            g[rr, cc] = v
            state.update(stats=stats, grad_logprob=g)
            if case.get("entropy"):
                ge = torch.zeros(rows, cols, **f32)
                ge[rr, cc] = -0.01 * torch.rand(rr.numel(), generator=gen, **f32)
                state.update(entropy=ent, grad_entropy=ge)
        if own:
            if kind == "grad":
                state["out"] = (torch.empty(rows, cols, V, dtype=logits.dtype, device=dev),)
            else:
                state["out"] = (torch.empty(rows, cols, **f32), torch.empty(rows, cols, 2, **f32),
                                torch.empty(rows, cols, **f32) if case.get("entropy") else None)
            state["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
        return state
    s, counted, gen = _tiles(case, seed)
    dev, E, n = counted.device, s["num_elems"], s["num_rows"]
    noise = lambda sd: torch.where(counted, torch.randn(E, generator=gen, device=dev) * sd,
                                   torch.zeros(E, device=dev))
    state.update(s)
    lp = _logprobs_like(counted, gen)
    state["logprob"] = lp
    K = s["slot_rows"].numel()
    if kind == "policy":
        state["old"] = lp + noise(0.15) if case.get("old", True) else None
        state["ref"] = lp + noise(0.3) if case["kl"] != "none" else None
        size = E if case.get("token_advantage") else n
        adv = torch.randn(size, generator=gen, device=dev)
        state["advantage"] = torch.where(torch.rand(size, generator=gen, device=dev) < 0.05, torch.zeros_like(adv), adv)
        state["entropy"] = torch.where(counted, torch.rand(E, generator=gen, device=dev) * 6.0,
                                       torch.zeros(E, device=dev)) if case.get("entropy") else None
        w = torch.rand(K, generator=gen, device=dev, dtype=torch.float64)
        state["slot_weight"] = w / w.sum()
    else:
        state["ref"] = lp + noise(0.3) if case.get("reference", True) else None
        # pairs of samples (or rows), either one chosen; an odd one out has none
        p = torch.randperm(n, generator=gen, device=dev)
        c, r = p[0:n // 2 * 2:2], p[1:n // 2 * 2:2]
        pair = torch.zeros(n, dtype=torch.int32, device=dev)
        pair[c] = (r + 1).int()
        pair[r] = -(c + 1).int()
        state["pair"] = pair
    if own:
        import paper_2606_19989_amd as odb

        f32 = dict(dtype=torch.float32, device=dev)
        t = odb.Tiles(s["slot_rows"], s["slot_maxlen"], s["slot_row_off"], s["slot_tile_off"], s["labels"], n)
        state["tiles"] = t
        state["ws"] = torch.empty(odb.odb_loss_workspace_size(t, 0 if kind == "policy" else n), dtype=torch.uint8,
                                  device=dev)
        if kind == "policy":
            state["out"] = (torch.empty(K, **f32), torch.empty(K, 4, **f32),
                            torch.empty(K, 4, dtype=torch.int64, device=dev), torch.empty(E, **f32),
                            torch.empty(E, **f32) if case.get("entropy") else None)
        else:
            state["out"] = (torch.empty(1, **f32), torch.empty(n, **f32), torch.empty(n, **f32),
                            torch.empty(2, dtype=torch.int64, device=dev), torch.empty(E, **f32))
        state["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    return state


# The loss parameters that the cases share.
CLIP_LOW, CLIP_HIGH, KL_COEF, ENTROPY_COEF, BETA = 0.2, 0.28, 0.04, 0.01, 0.1


def _loss_scale(case):
    return 8.0 if case["kind"] == "policy" else 1.0 / 64


# ---------------------------------------------------------------------- the plain forms
def _blocks(n, vocab):
    """Runs of positions whose logits make at most 2^27 values."""
    step = max(1, (1 << 27) // vocab)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _scored(labels, shift):
    c = torch.arange(labels.shape[1], device=labels.device)
    rr, cc = torch.nonzero((labels != IGNORE) & (c[None, :] >= shift), as_tuple=True)
    return rr, cc, labels[rr, cc].long()


def _plain_logprobs(s):
    case, z_all, a = s["case"], s["logits"], s["scale"]
    rows, cols, V = z_all.shape
    rr, cc, y = _scored(s["labels"], case["shift"])
    f32 = dict(dtype=torch.float32, device=z_all.device)
    out = {"logprob": torch.zeros(rows, cols, **f32), "stats": torch.zeros(rows, cols, 2, **f32)}
    if case.get("entropy"):
        out["entropy"] = torch.zeros(rows, cols, **f32)
    for i, j in _blocks(rr.numel(), V):
        r, c = rr[i:j], cc[i:j]
        z = z_all[r, c - case["shift"]].float()
        m = z.max(dim=-1, keepdim=True).values
        x = a * (z - m)
        e = torch.exp(x)
        total = e.sum(-1, keepdim=True)
        lse = torch.log(total)
        out["logprob"][r, c] = (x.gather(-1, y[i:j, None]) - lse)[:, 0]
        out["stats"][r, c] = torch.cat([m, lse], -1)
        if case.get("entropy"):
            ex = torch.where(e > 0, e * x, torch.zeros_like(x))
            out["entropy"][r, c] = (lse - ex.sum(-1, keepdim=True) / total)[:, 0]
    return out


def _plain_grad(s):
    case, z_all, a = s["case"], s["logits"], s["scale"]
    rows, cols, V = z_all.shape
    rr, cc, y = _scored(s["labels"], case["shift"])
    out = torch.zeros(rows, cols, V, dtype=z_all.dtype, device=z_all.device)
    for i, j in _blocks(rr.numel(), V):
        r, c = rr[i:j], cc[i:j]
        st = s["stats"][r, c]
        logp = a * (z_all[r, c - case["shift"]].float() - st[:, :1]) - st[:, 1:]
        p = torch.exp(logp)
        g = s["grad_logprob"][r, c][:, None]
        d = -g * p
        if case.get("entropy"):
            d = d - s["grad_entropy"][r, c][:, None] * torch.where(p > 0, p * (logp + s["entropy"][r, c][:, None]),
                                                                  torch.zeros_like(p))
        # g (1 - p) in one place, so that nothing cancels there
        at = y[i:j, None]
        d = d.scatter(-1, at, d.gather(-1, at) + g)
        out[r, c - case["shift"]] = (a * d).to(z_all.dtype)
    return out


def _maps(s):
    """Row and column of every element of the tiles."""
    rows, maxlen = s["slot_rows"].long(), s["slot_maxlen"].long()
    dev = rows.device
    row_max = torch.repeat_interleave(maxlen, rows)
    start = torch.cumsum(row_max, 0) - row_max
    row = torch.repeat_interleave(torch.arange(row_max.numel(), device=dev), row_max)
    return row, torch.arange(s["num_elems"], device=dev) - start[row]


def _runs(x, ends):
    """Sums over consecutive runs, in 64 bits; `ends` are the runs' last positions + 1."""
    lengths = ends - torch.cat([ends.new_zeros(1), ends[:-1]])
    return torch.segment_reduce(x.double(), "sum", lengths=lengths, initial=0.0, unsafe=True).to(x.dtype)


def _plain_policy(s):
    case = s["case"]
    row, col = _maps(s)
    E, K = s["num_elems"], s["slot_rows"].numel()
    slot = torch.repeat_interleave(torch.arange(K, device=row.device), s["slot_rows"].long() * s["slot_maxlen"].long())
    on = (s["labels"] != IGNORE) & (col >= 1)
    lp = s["logprob"]
    A = s["advantage"] if case.get("token_advantage") else s["advantage"][row]
    d = torch.zeros(E, dtype=torch.float64, device=row.device)
    if s["old"] is not None:
        d = lp.double() - s["old"].double()
    ratio = torch.exp(d.float())
    high = on & (A > 0) & (d > math.log1p(CLIP_HIGH))
    low = on & (A < 0) & (d < math.log1p(-CLIP_LOW))
    dual = on & (A < 0) & (d > (math.log(case["dual_clip"]) if case.get("dual_clip") else math.inf))
    loss = -ratio * A
    loss = torch.where(high, -(1 + CLIP_HIGH) * A, loss)
    loss = torch.where(low, -(1 - CLIP_LOW) * A, loss)
    loss = torch.where(dual, -case.get("dual_clip", 0.0) * A, loss)
    grad = torch.where(high | low | dual, torch.zeros_like(A), -ratio * A)
    kl, kl_grad = torch.zeros_like(lp), torch.zeros_like(lp)
    if case["kl"] != "none":
        x = lp.double() - s["ref"].double()    # in 64 bits: e^-x + x - 1 cancels for small x
        if case["kl"] == "linear":
            kl, kl_grad = x, torch.ones_like(x)
        elif case["kl"] == "square":
            kl, kl_grad = x * x / 2, x
        else:
            kl, kl_grad = torch.exp(-x) + x - 1, 1 - torch.exp(-x)
        kl, kl_grad = kl.float(), kl_grad.float()
    # weight of each counted token in its slot's reduction
    tile_end = s["slot_tile_off"][1:]
    row_max = torch.repeat_interleave(s["slot_maxlen"].long(), s["slot_rows"].long())
    count = _runs(on.long(), tile_end)
    if case["reduce"] == "token_mean":
        weight = 1.0 / count.clamp(min=1).double()[slot]
    elif case["reduce"] == "row_mean":
        per_row = _runs(on.long(), torch.cumsum(row_max, 0))
        rows = _runs((per_row > 0).long(), s["slot_row_off"][1:])
        weight = 1.0 / (per_row.clamp(min=1)[row].double() * rows.clamp(min=1)[slot].double())
    else:
        weight = torch.ones(E, dtype=torch.float64, device=row.device)
    weight = torch.where(on, weight, torch.zeros_like(weight))
    H = s["entropy"] if s["entropy"] is not None else torch.zeros_like(lp)
    mean = lambda v: _runs(torch.where(on, v.double() * weight, torch.zeros_like(weight)), tile_end)
    means = [mean(loss), mean(kl), mean(H), mean(ratio)]
    slot_scale = _loss_scale(case) * s["slot_weight"]
    total = means[0] + KL_COEF * means[1] - (ENTROPY_COEF if case.get("entropy") else 0.0) * means[2]
    scale = weight * slot_scale[slot]
    out = {"slot_loss": (slot_scale * total).float(), "slot_means": torch.stack(means, 1).float(),
           "slot_counts": torch.stack([count] + [_runs(v.long(), tile_end) for v in (low, high, dual)], 1),
           "grad_logprob": torch.where(on, scale * (grad.double() + KL_COEF * kl_grad.double()),
                                       torch.zeros_like(scale)).float()}
    if case.get("entropy"):
        out["grad_entropy"] = (-ENTROPY_COEF * scale).float()
    return out


def _partner_rows(s):
    """Row of each row's partner (-1: none here), and whether the row is the chosen one."""
    n, dev = s["num_rows"], s["pair"].device
    if not s["case"].get("ids"):
        v = s["pair"].long()
        return v.abs() - 1, v > 0
    ids = s["row_ids"].long()
    row_of = torch.full((s["pair"].numel(),), -1, dtype=torch.int64, device=dev)
    row_of[ids] = torch.arange(n, device=dev)
    v = s["pair"][ids].long()
    return torch.where(v != 0, row_of[(v.abs() - 1).clamp(min=0)], -torch.ones_like(v)), v > 0


def _plain_preference(s):
    case = s["case"]
    row, col = _maps(s)
    on = (s["labels"] != IGNORE) & (col >= 1)
    x = s["logprob"].double()
    if s["ref"] is not None:
        x = x - s["ref"].double()
    row_end = torch.cumsum(torch.repeat_interleave(s["slot_maxlen"].long(), s["slot_rows"].long()), 0)
    S = _runs(torch.where(on, x, torch.zeros_like(x)), row_end)
    count = _runs(on.long(), row_end)
    per = torch.ones_like(S)
    if case.get("normalize"):
        per = 1.0 / count.clamp(min=1).double()
    S = S * per
    partner, chosen = _partner_rows(s)
    paired = partner >= 0
    T = S[partner.clamp(min=0)]
    h = torch.where(chosen, S - T, T - S) * BETA - case.get("margin", 0.0)
    scale, eps = _loss_scale(case), case.get("smoothing", 0.0)
    soft = lambda v: torch.log1p(torch.exp(-v.abs())) + v.clamp(min=0)      # -log sigmoid(-v)
    if case["loss"] == "sigmoid":
        loss, dh = (1 - eps) * soft(-h) + eps * soft(h), eps - 1 / (1 + torch.exp(h))
    elif case["loss"] == "hinge":
        loss, dh = (1 - h).clamp(min=0), -(h < 1).double()
    else:
        loss, dh = ((h - 0.5) / BETA) ** 2, 2 * (h - 0.5) / BETA ** 2
    zero = torch.zeros_like(loss)
    row_loss = torch.where(paired & chosen, scale * loss, zero)
    coef = torch.where(paired, scale * BETA * torch.where(chosen, dh, -dh) * per, zero)
    return {"loss": row_loss.sum().float().reshape(1), "row_loss": row_loss.float(), "row_reward": (BETA * S).float(),
            "counts": torch.stack([(paired & chosen).sum(), (paired & chosen & (S > T)).sum()]),
            "grad_logprob": torch.where(on, coef[row], torch.zeros_like(x)).float()}


# ------------------------------------------------------------------------------- a pass
def _own(s):
    import paper_2606_19989_amd as odb

    case, out = s["case"], s["out"]
    kind = case["kind"]
    if kind == "logprobs":
        lp, stats, ent = out
        odb.odb_token_logprobs(s["logits"], s["labels"], lp, stats=stats, entropy=ent, status=s["status"],
                               shift=case["shift"], scale=s["scale"])
        res = {"logprob": lp, "stats": stats}
        if ent is not None:
            res["entropy"] = ent
        return res
    if kind == "grad":
        odb.odb_token_logprobs_backward(s["logits"], s["labels"], s["stats"], s["grad_logprob"], out[0],
                                        entropy=s.get("entropy"), grad_entropy=s.get("grad_entropy"),
                                        status=s["status"], shift=case["shift"], scale=s["scale"])
        return out[0]
    if kind == "policy":
        loss, means, counts, g, ge = out
        p = odb.PolicyParams(kl=KL[case["kl"]], reduce=REDUCE[case["reduce"]],
                             token_advantage=int(case.get("token_advantage", False)), clip_low=CLIP_LOW,
                             clip_high=CLIP_HIGH, dual_clip=case.get("dual_clip", 0.0), kl_coef=KL_COEF,
                             entropy_coef=ENTROPY_COEF if case.get("entropy") else 0.0, loss_scale=_loss_scale(case))
        odb.odb_policy_loss(s["tiles"], p, s["logprob"], s["advantage"], loss, means, counts, s["ws"],
                            old_logprob=s["old"], ref_logprob=s["ref"], entropy=s["entropy"],
                            slot_weight=s["slot_weight"], grad_logprob=g, grad_entropy=ge, status=s["status"])
        res = {"slot_loss": loss, "slot_means": means, "slot_counts": counts, "grad_logprob": g}
        if ge is not None:
            res["grad_entropy"] = ge
        return res
    loss, row_loss, reward, counts, g = out
    p = odb.PreferenceParams(kind=PREFERENCE[case["loss"]], normalize=int(case.get("normalize", False)), beta=BETA,
                             margin=case.get("margin", 0.0), label_smoothing=case.get("smoothing", 0.0),
                             loss_scale=_loss_scale(case))
    odb.odb_preference_loss(s["tiles"], p, s["logprob"], s["pair"], loss, row_loss, reward, counts, s["ws"],
                            ref_logprob=s["ref"], row_ids=s["row_ids"] if case.get("ids") else None, grad_logprob=g,
                            status=s["status"])
    return {"loss": loss, "row_loss": row_loss, "row_reward": reward, "counts": counts, "grad_logprob": g}


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "grad": _plain_grad, "policy": _plain_policy,
            "preference": _plain_preference}[state["case"]["kind"]](state)


def work(case):
    """Each input read once and each output written once; about what the formulas compute."""
    if case["kind"] in ("logprobs", "grad"):
        tokens = case["rows"] * case["cols"]
        scored = int(_counted_rows(case).sum())
        row = case["vocab"] * _BYTES[case["dtype"]]
        ent = bool(case.get("entropy"))
        if case["kind"] == "logprobs":
            return {"bytes": scored * row + tokens * (16 + 4 * ent), "flops": scored * case["vocab"] * (4 + 2 * ent)}
        read = scored * (1.0 - (0.0 if ent else case.get("zeros", 0.0)))
        return {"bytes": int(read * row) + tokens * row + tokens * (16 + 8 * ent),
                "flops": int(read) * case["vocab"] * (4 + 4 * ent)}
    E, n = case["elems"], max(2, case["elems"] // case["mean_len"])
    slots = max(1, E // case["budget"]) if case["budget"] else 1
    if case["kind"] == "policy":
        per = 12 + 4 * case.get("old", True) + 4 * (case["kl"] != "none") + 8 * bool(case.get("entropy")) \
            + 4 * bool(case.get("token_advantage"))
        return {"bytes": E * per + 4 * n + slots * (24 + 8 + 52), "flops": 20 * E}
    return {"bytes": E * (12 + 4 * case.get("reference", True)) + n * (12 + 4 * bool(case.get("ids"))) + 24 * slots,
            "flops": 4 * E}


# ------------------------------------------------------------------ the outputs in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "grad": _exact_grad, "policy": _exact_policy,
            "preference": _exact_preference}[case["kind"]](state)


def _log_softmax64(s, i, j, rr, cc):
    """Log-probabilities of a run of scored positions, from the definition."""
    z = s["logits"][rr[i:j], cc[i:j] - s["case"]["shift"]].double()
    return z, z * s["scale"] - torch.logsumexp(z * s["scale"], -1, keepdim=True)


def _exact_logprobs(s):
    rr, cc, y = _scored(s["labels"], s["case"]["shift"])
    rows, cols, V = s["logits"].shape
    f64 = dict(dtype=torch.float64, device=s["logits"].device)
    out = {"logprob": torch.zeros(rows, cols, **f64), "stats": torch.zeros(rows, cols, 2, **f64)}
    if s["case"].get("entropy"):
        out["entropy"] = torch.zeros(rows, cols, **f64)
    for i, j in _blocks(rr.numel(), 2 * V):
        z, lq = _log_softmax64(s, i, j, rr, cc)
        out["logprob"][rr[i:j], cc[i:j]] = lq.gather(-1, y[i:j, None])[:, 0]
        top, at = z.max(-1)
        out["stats"][rr[i:j], cc[i:j], 0] = top
        out["stats"][rr[i:j], cc[i:j], 1] = -lq.gather(-1, at[:, None])[:, 0]
        if "entropy" in out:
            out["entropy"][rr[i:j], cc[i:j]] = torch.special.entr(lq.exp()).sum(-1)
    return out


def _exact_grad(s):
    rr, cc, y = _scored(s["labels"], s["case"]["shift"])
    rows, cols, V = s["logits"].shape
    out = torch.zeros(rows, cols, V, dtype=torch.float64, device=s["logits"].device)
    for i, j in _blocks(rr.numel(), 2 * V):
        _, lq = _log_softmax64(s, i, j, rr, cc)
        q = lq.exp()
        g = s["grad_logprob"][rr[i:j], cc[i:j]].double()[:, None]
        d = g * (torch.zeros_like(q).scatter_(-1, y[i:j, None], 1.0) - q)
        if s["case"].get("entropy"):
            ge = s["grad_entropy"][rr[i:j], cc[i:j]].double()[:, None]
            info = torch.special.entr(q)                       # -q ln q
            d = d + ge * (info - q * info.sum(-1, keepdim=True))
        out[rr[i:j], cc[i:j] - s["case"]["shift"]] = s["scale"] * d
    return out


def _sum_by(v, at, n):
    return torch.zeros(n, dtype=v.dtype, device=v.device).index_add_(0, at, v)


def _exact_policy(s):
    """The definition with min and clamp over the counted tokens alone; gradients by differentiation."""
    case = s["case"]
    row, col = _maps(s)
    K, E = s["slot_rows"].numel(), s["num_elems"]
    at = torch.nonzero((s["labels"] != IGNORE) & (col >= 1))[:, 0]
    slot_of_row = torch.repeat_interleave(torch.arange(K, device=row.device), s["slot_rows"].long())
    row = row[at]
    slot = slot_of_row[row]
    one = torch.ones(at.numel(), dtype=torch.float64, device=row.device)
    n_slot, n_row = _sum_by(one, slot, K), _sum_by(one, row, s["num_rows"])
    n_rows = _sum_by((n_row > 0).double(), slot_of_row, K)
    w = {"token_mean": lambda: 1 / n_slot[slot], "row_mean": lambda: 1 / (n_row[row] * n_rows[slot]),
         "sum": lambda: one}[case["reduce"]]()
    lp = s["logprob"][at].double().requires_grad_()
    old = lp.detach() if s["old"] is None else s["old"][at].double()
    A = (s["advantage"][at] if case.get("token_advantage") else s["advantage"][row]).double()
    r = (lp - old).exp()
    pg = -torch.minimum(r * A, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
    if case.get("dual_clip"):
        pg = torch.where(A < 0, torch.minimum(pg, -case["dual_clip"] * A), pg)
    kl = torch.zeros_like(r)
    if s["ref"] is not None:
        x = lp - s["ref"][at].double()
        kl = {"linear": lambda: x, "square": lambda: 0.5 * x ** 2, "exp": lambda: torch.expm1(-x) + x}[case["kl"]]()
    H = torch.zeros_like(one)
    if s["entropy"] is not None:
        H = s["entropy"][at].double().requires_grad_()
    c_ent = ENTROPY_COEF if s["entropy"] is not None else 0.0
    scale = s["slot_weight"] * _loss_scale(case)
    loss = _sum_by(w * (pg + KL_COEF * kl - c_ent * H), slot, K) * scale
    grads = torch.autograd.grad(loss.sum(), [lp] + ([H] if s["entropy"] is not None else []))
    full = lambda g: torch.zeros(E, dtype=torch.float64, device=g.device).index_copy_(0, at, g)
    out = {"slot_loss": loss.detach(),
           "slot_means": torch.stack([_sum_by(w * v.detach(), slot, K) for v in (pg, kl, H, r)], 1),
           "slot_counts": None, "grad_logprob": full(grads[0])}
    if s["entropy"] is not None:
        out["grad_entropy"] = full(grads[1])
    return out


def _exact_preference(s):
    case = s["case"]
    row, col = _maps(s)
    at = torch.nonzero((s["labels"] != IGNORE) & (col >= 1))[:, 0]
    row = row[at]
    n = s["num_rows"]
    lp = s["logprob"][at].double().requires_grad_()
    x = lp if s["ref"] is None else lp - s["ref"][at].double()
    S = _sum_by(x, row, n)
    if case.get("normalize"):
        S = S / _sum_by(torch.ones_like(x), row, n).clamp(min=1).detach()
    # the pairs one by one, chosen first, in rows
    pair = s["pair"].long()
    chosen = torch.nonzero(pair > 0)[:, 0]
    other = pair[chosen] - 1
    if case.get("ids"):
        row_of = torch.empty_like(pair)
        row_of[s["row_ids"].long()] = torch.arange(n, device=pair.device)
        chosen, other = row_of[chosen], row_of[other]
    h = BETA * (S[chosen] - S[other]) - case.get("margin", 0.0)
    eps = case.get("smoothing", 0.0)
    logsig = torch.nn.functional.logsigmoid
    loss = {"sigmoid": lambda: -(1 - eps) * logsig(h) - eps * logsig(-h), "hinge": lambda: torch.relu(1 - h),
            "square": lambda: ((h - 0.5) / BETA) ** 2}[case["loss"]]() * _loss_scale(case)
    g, = torch.autograd.grad(loss.sum(), [lp])
    zeros = lambda k: torch.zeros(k, dtype=torch.float64, device=g.device)
    return {"loss": loss.detach().sum().reshape(1), "row_loss": zeros(n).index_copy_(0, chosen, loss.detach()),
            "row_reward": (BETA * S).detach(), "counts": None,
            "grad_logprob": zeros(s["num_elems"]).index_copy_(0, at, g)}
