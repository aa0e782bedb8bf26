"""The likeliest tokens where a block takes a position and goes through many rounds of it: its waves go on by themselves
once they have a bound, form it anew in some rounds only, and look at what they set aside under the last one.  And the
gradient of lists, the same bit for bit from call to call."""
import math

import numpy as np
import pytest

from _losses import IGNORE
from _parity import log
from test_gpu_lists import _check_top, _dev, _hard_rows, _top, _types

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


@pytest.mark.parametrize("k", [20, 64, 128])
@pytest.mark.parametrize("V,dtype", [(50003, "fp32"), (152001, "bf16"), (70001, "fp16")])
def test_top_of_hard_rows_by_a_block(V, dtype, k):
    """More positions than are split (1,024 / 2): 13, 19 and 9 rounds of a block, cells of threads (k up to 64) and of
    half groups; every row many times, of which two are compared with the oracle and all with each other."""
    torch = _torch()
    rows = _hard_rows(V, np.random.default_rng(V))
    rng = np.random.default_rng(2)
    rows["random"] = (rng.standard_normal(V) * 2.5).astype(np.float32)
    names = list(rows)
    z = torch.from_numpy(np.stack([rows[n] for n in names]))
    if dtype != "fp32":
        limit = torch.finfo(_types()[dtype])
        z = z.clamp(min=limit.min, max=limit.max)
        z[names.index("three finite")][z[names.index("three finite")] < -1e4] = -math.inf
    z = z.to(_types()[dtype])
    z64 = z.double().numpy()[:, None]
    copies = 520 // len(names) + 1
    assert copies * len(names) > 512
    zd = z.cuda()[:, None].repeat(copies, 1, 1)
    y = rng.integers(0, V, (len(names), 1)).astype(np.int32)
    y[names.index("three finite")] = V // 2
    on = np.ones((len(names), 1), bool)
    for rank, entropy in ((True, True), (True, False), (False, True), (False, False)):
        log(f"top by a block: {V} {dtype}, k {k}, rank {rank}, entropy {entropy}")
        o = _top(zd, k, _dev(np.tile(y, (copies, 1))), rank=rank, entropy=entropy)
        o = {n: v for n, v in o.items() if v is not None}
        first = {n: v[:len(names)] for n, v in o.items()}
        for n, v in o.items():
            assert np.array_equal(v, np.tile(first[n], (copies,) + (1,) * (v.ndim - 1)), equal_nan=True), n
        for i, name in enumerate(names):
            log(f"  {name}")
            one = {n: first[n][i:i + 1] if n in first else None for n in ("ids", "top", "stats", "entropy", "logprob", "rank")}
            one["entropy"] = None if name == "huge" else one["entropy"]
            _check_top(one, z64[i:i + 1], y[i:i + 1], on[i:i + 1], k, 0, 1.0, 4 if dtype == "fp32" else 2)


@pytest.mark.parametrize("V,k", [(500, 128), (4096, 100), (9001, 128)])
def test_gradient_of_lists_with_shared_ids_from_call_to_call(V, k):
    import paper_2606_19989_amd as odb
    torch = _torch()
    gen = torch.Generator("cuda").manual_seed(V)
    z = torch.randn(40, 9, V, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, 60, (40, 9, k), generator=gen, device="cuda", dtype=torch.int32)      # most of them twice or more
    ids[:, :, 5] = IGNORE
    out, st = torch.empty(40, 9, k, device="cuda"), torch.empty(40, 9, 2, device="cuda")
    odb.odb_token_list_logprobs(z, ids, out, stats=st)
    g = torch.randn(40, 9, k, generator=gen, device="cuda")
    first = None
    for _ in range(4):
        d = torch.full_like(z, 5.0)
        odb.odb_token_list_logprobs_backward(z, ids, st, g, d)
        first = d if first is None else first
        assert torch.equal(d, first)
