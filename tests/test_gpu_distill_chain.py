"""The operators over lists used together: what a teacher keeps, a student's log-probabilities of it, the loss over
a plan's tiles, the gradient back at the student's logits; in graphs, on streams, past 32 bits and past a grid."""
import math

import numpy as np
import pytest

import _lists as ref
import synth
from _losses import IGNORE, U
from _parity import log

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


# ------------------------------------------------------------------ one tile's step
OUTPUTS = ("ids", "top", "tst", "rank", "lst", "sst", "loss", "mean", "count", "gs", "dz")
INPUTS = ("zt", "zs", "y")


def _state(rows, cols, V, k, seed, support=1, reduce=0):
    import paper_2606_19989_amd as odb
    torch = _torch()
    gen = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *n: torch.randn(*n, generator=gen, device="cuda")
    f32, i32, i64 = (dict(dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int64))
    s = {"zt": (rnd(rows, cols, V) * 3).bfloat16(), "zs": (rnd(rows, cols, V) * 3).bfloat16(), "k": k, "stream": None}
    s["y"] = torch.randint(0, V, (rows, cols), generator=gen, **i32)
    s["y"][rnd(rows, cols) < -0.5] = IGNORE
    s.update(ids=torch.empty(rows, cols, k, **i32), top=torch.empty(rows, cols, k, **f32), tst=torch.empty(rows, cols, 2, **f32),
             rank=torch.empty(rows, cols, **i32), lst=torch.empty(rows, cols, k, **f32), sst=torch.empty(rows, cols, 2, **f32),
             loss=torch.empty(1, **f32), mean=torch.empty(1, **f32), count=torch.empty(1, **i64),
             gs=torch.empty(rows, cols, k, **f32), dz=torch.empty(rows, cols, V, dtype=torch.bfloat16, device="cuda"))
    one = lambda v, t: torch.tensor(v, **t)
    s["tiles"] = odb.Tiles(one([rows], i32), one([cols], i32), one([0, rows], i64), one([0, rows * cols], i64),
                           s["y"].view(-1), rows)
    s["params"] = odb.DistillParams(support=support, reduce=reduce, loss_scale=3.0)
    s["tws"] = torch.empty(odb.odb_token_top_workspace_size(s["zt"], k), dtype=torch.uint8, device="cuda")
    s["ws"] = torch.empty(odb.odb_distill_workspace_size(s["tiles"], k), dtype=torch.uint8, device="cuda")
    s["status"] = torch.zeros(1, **i32)
    return s


def _step(s):
    import paper_2606_19989_amd as odb
    st, k = s["stream"], s["k"]
    odb.odb_token_top_logprobs(s["zt"], s["ids"], s["top"], s["tws"], labels=s["y"], rank=s["rank"], stats=s["tst"],
                               status=s["status"], stream=st)
    odb.odb_token_list_logprobs(s["zs"], s["ids"], s["lst"], labels=s["y"], stats=s["sst"], status=s["status"], stream=st)
    odb.odb_distill_loss(s["tiles"], s["params"], s["lst"].view(-1, k), s["top"].view(-1, k), s["loss"], s["mean"],
                         s["count"], s["ws"], grad_student=s["gs"].view(-1, k), status=s["status"], stream=st)
    odb.odb_token_list_logprobs_backward(s["zs"], s["ids"], s["sst"], s["gs"], s["dz"], labels=s["y"], status=s["status"],
                                         stream=st)


# one block's loss; parts of a position and the passes; a wave a position
SHAPES = [(3, 9, 50, 5), (2, 5, 60000, 20), (6, 300, 3000, 64)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step_in_a_graph_and_on_streams(shape):
    torch = _torch()
    log(f"distillation step in a graph {shape}")
    s = _state(*shape, seed=1)
    other = _state(*shape, seed=2, support=2, reduce=1)
    eager = {}
    for seed in (1, 3, 4):
        v = _state(*shape, seed=seed)
        _step(v)
        eager[seed] = {n: v[n].clone() for n in OUTPUTS + INPUTS}
        assert int(v["status"].item()) == 0
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        _step(s)          # loads the kernels
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        _step(s)
    for seed in (3, 1, 4, 1):
        for n in INPUTS:
            s[n].copy_(eager[seed][n])
        for n in OUTPUTS:
            s[n].zero_()
        torch.cuda.synchronize()
        _step(other)      # eager work with workspaces of its own between the replays
        graph.replay()
        torch.cuda.synchronize()
        for n in OUTPUTS:
            assert torch.equal(s[n], eager[seed][n]), (seed, n)
    # two streams at once, each with its own workspaces
    a, b = _state(*shape, seed=3), _state(*shape, seed=4)
    torch.cuda.synchronize()
    a["stream"], b["stream"] = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        _step(a)
        _step(b)
    torch.cuda.synchronize()
    for n in OUTPUTS:
        assert torch.equal(a[n], eager[3][n]) and torch.equal(b[n], eager[4][n]), n


# ------------------------------------------------------------------ behind a window
@pytest.mark.parametrize("support", [0, 1, 2])
def test_chain_behind_a_window(support):
    """Collate, a teacher's and a student's logits per tile, the loss over the whole plan with its loss weights, the
    gradient back per tile; again in 64 bits by torch's differentiation."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(81 + support)
    W, V, k = 3, 61, 7
    w = synth.window_from_ranks("distill_chain", [rng.integers(2, 60, 40) for _ in range(W)], 400)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")
    pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
    pipe.form()
    pipe.align()
    labels = pipe.collate()[1]
    K, P = pipe.num_slots, int(pipe.info["padded_elems"])
    log(f"distillation behind a window: {K} slots, {P} elements")
    labels.copy_(torch.where(labels != IGNORE, labels % V, labels))       # the tiny models' vocabulary
    rows, maxlen = pipe.slot_rows[:K].tolist(), pipe.slot_maxlen[:K].tolist()
    off = pipe.slot_tile_off[:K + 1].tolist()
    tile = lambda x, j: x[off[j]:off[j + 1]].view(rows[j], maxlen[j], *x.shape[1:])
    gen = torch.Generator("cuda").manual_seed(81)
    zt, zs = (torch.randn(P, V, generator=gen, device="cuda") * 2 for _ in range(2))
    f32 = dict(dtype=torch.float32, device="cuda")
    ids = torch.empty(P, k, dtype=torch.int32, device="cuda")
    top, lst, st = torch.empty(P, k, **f32), torch.empty(P, k, **f32), torch.empty(P, 2, **f32)
    scale = 0.8
    for j in range(K):
        if rows[j]:
            ws = torch.empty(odb.odb_token_top_workspace_size(tile(zt, j), k), dtype=torch.uint8, device="cuda")
            odb.odb_token_top_logprobs(tile(zt, j), tile(ids, j), tile(top, j), ws, labels=tile(labels, j), scale=scale)
            odb.odb_token_list_logprobs(tile(zs, j), tile(ids, j), tile(lst, j), labels=tile(labels, j),
                                        stats=tile(st, j), scale=scale)
    tiles = pipe.tiles(labels)
    weight = pipe.loss_weights(odb.ODB_WEIGHT_TOKEN_EXACT)[0]
    params = odb.DistillParams(kind=odb.ODB_DISTILL_FORWARD, support=support, reduce=odb.ODB_REDUCE_TOKEN_MEAN,
                               loss_scale=float(W))
    loss, mean, count, g = pipe.distill_loss(tiles, lst, top, params, weight)
    dz = torch.full((P, V), 9.0, **f32)
    for j in range(K):
        if rows[j]:
            odb.odb_token_list_logprobs_backward(tile(zs, j), tile(ids, j), tile(st, j), tile(g, j), tile(dz, j),
                                                 labels=tile(labels, j), scale=scale)
    pipe.check_losses()

    x = zs.double().cpu().requires_grad_()
    t64, y = zt.double().cpu(), labels.cpu()
    total = torch.zeros((), dtype=torch.float64)
    for j in range(K):
        if not rows[j]:
            assert float(loss[j]) == 0 and int(count[j]) == 0
            continue
        on = tile(y, j)[:, 1:] != IGNORE
        lt = torch.log_softmax(scale * tile(t64, j)[:, :-1], -1)
        ls = torch.log_softmax(scale * tile(x, j)[:, :-1], -1)
        at = torch.from_numpy(np.argsort(-tile(t64, j)[:, :-1].numpy(), axis=-1, kind="stable")[..., :k].copy())
        assert torch.equal(tile(ids, j)[:, 1:].cpu()[on].long(), at[on])
        lt, ls = lt.gather(-1, at), ls.gather(-1, at)
        if support == 1:
            lt, ls = lt - torch.logsumexp(lt, -1, keepdim=True), ls - torch.logsumexp(ls, -1, keepdim=True)
        D = (lt.exp() * (lt - ls)).sum(-1)
        if support == 2:
            rp, rq = 1 - lt.exp().sum(-1), 1 - ls.exp().sum(-1)
            D = D + rp * (rp.log() - rq.log())
        n = int(on.sum())
        assert int(count[j]) == n
        want = float(weight[j]) * W * D[on].sum() / max(n, 1)
        # about 20 roundings of logs of size 20 on each side
        assert abs(float(loss[j]) - float(want.detach())) <= 800 * U * abs(float(weight[j])) * W * 2, j
        total = total + want
    want, = torch.autograd.grad(total, x)
    # per token: the slopes' sizes sum to 4 at most with renormalised lists or rests (p and q each sum to 1, once with
    # the sum's share), their logs are right to 400 U, and where the student's rest r is small its share to 400 U / r
    with torch.no_grad():
        share = torch.zeros(P, dtype=torch.float64)
        for j in range(K):
            if rows[j]:
                n = max(int(count[j]), 1)
                share[off[j]:off[j + 1]] = W * abs(float(weight[j])) / n
        rq = 1.0
        if support == 2:
            q = torch.exp(lst.double().cpu()).sum(-1)
            rq = (1 - q).clamp(min=2.0 ** -24)
            rq[(labels.cpu() == IGNORE)] = 1.0
        tol = 4 * 800 * U * share / rq
    err = (dz.double().cpu() - want).abs().amax(-1)
    assert bool((err <= tol + 1e-30).all()), float((err / (tol + 1e-30)).max())
    # tile by tile, as ranks call it: the same numbers as the whole plan's
    for j in (0, K - 1, K // 2):
        t = pipe.tiles(labels, first=j, count=1)
        keep = g[t.elems].clone(), loss[j].clone()
        one = pipe.distill_loss(t, lst[t.elems], top[t.elems], params, weight[t.slots])
        assert abs(float(one[0][0]) - float(keep[1])) <= 4 * U * abs(float(keep[1]))
        assert torch.allclose(one[3], keep[0], rtol=4 * U, atol=0)
        loss, mean, count, g = pipe.distill_loss(tiles, lst, top, params, weight)


def test_lists_with_the_label_behind_them():
    """A list one entry longer, the label in it with no teacher's share: the distillation's gradient and a label's in
    one call."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    s = _state(4, 12, 900, 6, seed=9)
    _step(s)
    y, k = s["y"], 6
    on = (y != IGNORE) & (torch.arange(12, device="cuda") >= 1)
    ids = torch.cat([s["ids"], y[..., None]], -1).contiguous()
    top = torch.cat([s["top"], torch.full_like(s["top"][..., :1], -math.inf)], -1).contiguous()
    lst, st = torch.empty(4, 12, k + 1, device="cuda"), torch.empty(4, 12, 2, device="cuda")
    odb.odb_token_list_logprobs(s["zs"], ids, lst, labels=y, stats=st)
    g = torch.empty(48, k + 1, device="cuda")
    ws = torch.empty(odb.odb_distill_workspace_size(s["tiles"], k + 1), dtype=torch.uint8, device="cuda")
    odb.odb_distill_loss(s["tiles"], s["params"], lst.view(48, k + 1), top.view(48, k + 1), s["loss"], s["mean"],
                         s["count"], ws, grad_student=g)
    assert torch.equal(g.view(4, 12, k + 1)[..., :k], s["gs"]) and bool((g[:, k] == 0).all())
    g.view(4, 12, k + 1)[..., k] = torch.where(on, -0.01, 0.0)
    both, label = torch.empty_like(s["zs"]), torch.empty_like(s["zs"])
    odb.odb_token_list_logprobs_backward(s["zs"], ids, st, g.view(4, 12, k + 1), both, labels=y)
    odb.odb_token_logprobs_backward(s["zs"], y, st, torch.full((4, 12), -0.01, device="cuda"), label)
    want = s["dz"].double() + label.double()
    # two roundings to bf16 of the parts, one of the sum
    assert bool(((both.double() - want).abs() <= 2.0 ** -8 * (s["dz"].double().abs() + label.double().abs() + want.abs())
                 + 64 * U).all())


def test_pipeline_distill_in_a_graph_and_growing():
    import paper_2606_19989_amd as odb
    torch = _torch()
    rng = np.random.default_rng(83)
    w = synth.window_from_ranks("distill_graph", [rng.integers(20, 90, 60)], 2000)
    tok_off, toks, ident = synth.device_tensors(w, "cuda")
    pipe = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
    pipe.form()
    pipe.align()
    pipe.collate()
    whole, part = pipe.tiles(), pipe.tiles(first=0, count=1)
    k = 9
    gen = torch.Generator("cuda").manual_seed(83)
    draw = lambda: torch.log_softmax(torch.randn(whole.num_elems, k + 3, generator=gen, device="cuda"), -1)[:, :k].contiguous()
    t, s = draw(), draw()
    params = odb.DistillParams(kind=2, support=1, reduce=1, mix=0.4)
    small = pipe.distill_loss(part, s[part.elems], t[part.elems], params)
    small = [v.clone() for v in small]
    big = [v.clone() for v in pipe.distill_loss(whole, s, t, params)]      # larger buffers
    assert torch.equal(small[0][0], big[0][0]) or abs(float(small[0][0]) - float(big[0][0])) <= 4 * U * abs(float(big[0][0]))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        pipe.distill_loss(whole, s, t, params)
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = pipe.distill_loss(whole, s, t, params)
    plain = odb.Pipeline(odb.DeviceWindow(w.rank_off, tok_off, toks, ident, w.num_identities), w.budget)
    plain.form()
    plain.align()
    plain.collate()
    other = plain.tiles()
    for _ in range(4):
        a, b = draw(), draw()
        t.copy_(a)
        s.copy_(b)
        want = plain.distill_loss(other, b, a, params)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, z) for x, z in zip(out, want))
    pipe.check_losses()
    bad = pipe.tiles()
    bad.keep[1][0] += 1
    pipe.distill_loss(bad, s, t, params)
    with pytest.raises(odb.OdbError):
        pipe.check_losses()


# ------------------------------------------------------------------ sizes
def test_logits_past_32_bits():
    """Rows that lie 2^31 elements apart, and a vocabulary's positions behind them."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    V, gap = 40003, (1 << 31) + 24
    log("lists: rows 2^31 elements apart")
    buf = torch.empty(gap + 2 * V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((2, 2, V), (gap, V, 1))
    z.copy_(torch.randn(2, 2, V, device="cuda") * 2)
    flat = z.contiguous()
    k = 33
    outs = []
    for x in (z, flat):
        ids = torch.empty(2, 2, k, dtype=torch.int32, device="cuda")
        top, st, lst = torch.empty(2, 2, k, device="cuda"), torch.empty(2, 2, 2, device="cuda"), torch.empty(2, 2, k, device="cuda")
        ws = torch.empty(odb.odb_token_top_workspace_size(x, k), dtype=torch.uint8, device="cuda")
        odb.odb_token_top_logprobs(x, ids, top, ws, stats=st, shift=0)
        odb.odb_token_list_logprobs(x, ids, lst, shift=0)
        outs.append((ids, top, st, lst))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    # the list's numbers and the alternatives' come from sums in another order
    assert float((outs[0][1] - outs[0][3]).abs().max()) <= 2 * U * (V / 256 + 100 + 30)
    g = torch.randn(2, 2, k, device="cuda")
    want = torch.empty_like(flat)
    odb.odb_token_list_logprobs_backward(flat, outs[0][0], outs[0][2], g, want, shift=0)
    odb.odb_token_list_logprobs_backward(z, outs[0][0], outs[0][2], g, z, shift=0)      # in place
    assert torch.equal(z, want)


def test_more_positions_than_a_grid_holds():
    """More than 2^20 blocks take at once: a position a block (one row of logits for all of them), and a wave."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    for n, V, k in ((1_060_003, 20000, 3), (4_300_003, 37, 2)):
        log(f"lists: {n} positions of {V}")
        z = torch.randn(1, 7, V, device="cuda", dtype=torch.float32).bfloat16()
        x = z[:, 2:3].expand(1, n, V)
        ids = torch.empty(1, n, k, dtype=torch.int32, device="cuda")
        top = torch.empty(1, n, k, device="cuda")
        ws = torch.empty(odb.odb_token_top_workspace_size(x, k), dtype=torch.uint8, device="cuda")
        y = torch.zeros(1, n, dtype=torch.int32, device="cuda")
        y[0, 5::11] = IGNORE
        odb.odb_token_top_logprobs(x, ids, top, ws, labels=y, shift=0)
        on = y[0] != IGNORE
        want = np.argsort(-z[0, 2].double().cpu().numpy(), kind="stable")[:k]
        assert bool((ids[0][on] == torch.from_numpy(want.copy()).cuda()).all()) and bool((ids[0][~on] == IGNORE).all())
        assert bool((top[0][on] == top[0, 0]).all()) and bool((top[0][~on] == -math.inf).all())
    n, V, k = 34_000_003, 5, 2
    log(f"lists: {n} positions of {V}")
    gen = torch.Generator("cuda").manual_seed(1)
    z = torch.randn(1, n, V, generator=gen, device="cuda").half()
    ids = torch.randint(0, V, (1, n, k), generator=gen, device="cuda", dtype=torch.int32)
    lst, st = torch.empty(1, n, k, device="cuda"), torch.empty(1, n, 2, device="cuda")
    odb.odb_token_list_logprobs(z, ids, lst, stats=st, shift=0)
    want = torch.log_softmax(z[0].double(), -1)
    assert float((lst[0].double() - want.gather(1, ids[0].long())).abs().max()) <= 32 * 20 * U
    g = torch.ones_like(lst)
    odb.odb_token_list_logprobs_backward(z, ids, st, g, z, shift=0)
    want = -2 * want.exp_()
    want.scatter_add_(1, ids[0].long(), torch.ones(n, k, dtype=torch.float64, device="cuda"))
    # rounded to fp16 (2^-11 of at most 2)
    assert float((z[0].double() - want).abs().max()) <= 2.0 ** -10 + 64 * U


def test_tiles_past_32_bits():
    """More than 2^31 elements in one slot of two rows: positions, the mean and the last elements."""
    import paper_2606_19989_amd as odb
    torch = _torch()
    L = (1 << 30) + 5
    E = 2 * L
    log(f"distillation past 32 bits: 2 x {L}")
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    y = torch.ones(E, **i32)
    y[L - 3:L] = IGNORE
    tiles = odb.Tiles(torch.tensor([2], **i32), torch.tensor([L], **i32), torch.tensor([0, 2], **i64),
                      torch.tensor([0, E], **i64), y, 2)
    ws = torch.empty(odb.odb_distill_workspace_size(tiles, 1), dtype=torch.uint8, device="cuda")
    t = torch.full((E, 1), math.log(0.5), device="cuda")
    s = torch.full((E, 1), math.log(0.25), device="cuda")
    grad = torch.full((E, 1), 7.0, device="cuda")
    loss, mean, count = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, **i64)
    status = torch.zeros(1, **i32)
    p, q = math.exp(np.float32(math.log(0.5))), math.exp(np.float32(math.log(0.25)))
    D = p * float(np.float32(math.log(0.5)) - np.float32(math.log(0.25)))
    a, b = L - 1 - 3, L - 1                     # counted tokens of the rows
    for reduce in (0, 1):
        odb.odb_distill_loss(tiles, odb.DistillParams(reduce=reduce, loss_scale=1e9), s, t, loss, mean, count, ws,
                             grad_student=grad, status=status)
        assert int(status.item()) == 0 and count.tolist() == [a + b]
        w0, w1 = (1 / (a + b), 1 / (a + b)) if reduce == 0 else (1 / (2 * a), 1 / (2 * b))
        assert abs(float(mean) - D) <= 16 * U * D and abs(float(loss) - 1e9 * D) <= 1e9 * 18 * U * D
        for at, w in ((0, 0.0), (1, w0), (L - 4, w0), (L - 3, 0.0), (L - 1, 0.0), (L, 0.0), (L + 1, w1), (E - 1, w1)):
            assert abs(float(grad[at, 0]) + 1e9 * w * p) <= 8 * U * 1e9 * w * p, at
        assert int((grad == 0).sum()) == 5


# ------------------------------------------------------------------ what the binding refuses
def test_binding_checks_types_sizes_and_streams():
    import paper_2606_19989_amd as odb
    torch = _torch()
    s = _state(4, 9, 50, 5, seed=1)
    _step(s)
    call = lambda **kw: odb.odb_token_top_logprobs(**{**dict(logits=s["zt"], top_ids=s["ids"], top_logprob=s["top"],
                                                             ws=s["tws"], labels=s["y"], rank=s["rank"]), **kw})
    for bad in (dict(top_ids=s["ids"].long()), dict(top_ids=s["ids"][:, :, :4]), dict(top_ids=s["ids"][:3]),
                dict(top_logprob=s["top"][:, :, :4]), dict(top_logprob=s["top"].half()), dict(rank=s["rank"].long()),
                dict(labels=s["y"].t()), dict(logits=s["zt"].double()), dict(ws=s["tws"].cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(odb.OdbError):
        call(ws=s["tws"][:8])
    with pytest.raises(odb.OdbError):
        call(labels=None)
    with pytest.raises(ValueError):
        odb.odb_token_list_logprobs(s["zs"], s["ids"], s["lst"][:, :, :3].contiguous())
    with pytest.raises(ValueError):
        odb.odb_token_list_logprobs_backward(s["zs"], s["ids"], s["sst"], s["gs"], s["dz"].float())
    with pytest.raises(ValueError):
        odb.odb_token_list_logprobs_backward(s["zs"], s["ids"], s["sst"], s["gs"], s["dz"][:, :, :40])
    flat = lambda n: s[n].view(-1, 5)
    loss = lambda **kw: odb.odb_distill_loss(**{**dict(tiles=s["tiles"], params=s["params"], student=flat("lst"),
                                                       teacher=flat("top"), slot_loss=s["loss"], slot_mean=s["mean"],
                                                       slot_count=s["count"], ws=s["ws"]), **kw})
    for bad in (dict(student=flat("lst")[:30]), dict(teacher=flat("top")[:, :4]), dict(student=flat("lst").double()),
                dict(teacher=flat("top")[:, :4].contiguous()), dict(student=s["loss"]),
                dict(grad_student=flat("gs").t().contiguous()), dict(slot_count=s["mean"]), dict(slot_weight=s["mean"]),
                dict(student=flat("lst").t().contiguous(), teacher=flat("top").t().contiguous())):
        with pytest.raises((ValueError, odb.OdbError)):
            loss(**bad)
    loss()
