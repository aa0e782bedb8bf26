"""The distillation loss over a run of 2^24 elements and more, whose chunks' counts are folded per slot before the pieces
add them up: slots of many chunks and of one, rows across hundreds of chunks and rows of one element."""
import numpy as np
import pytest

from _losses import IGNORE, U
from _parity import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reduce", [0, 1])
def test_folded_counts(reduce):
    import torch
    import paper_2606_19989_amd as odb
    rows, cols = [3000, 5000, 0, 2, 3], [3001, 1, 0, 4_000_003, 7]
    size = np.array(rows, np.int64) * cols
    E, R, K = int(size.sum()), sum(rows), len(rows)
    assert E >= 1 << 24
    log(f"distillation, counts folded: {E} elements in {K} slots, reduce {reduce}")
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    gen = torch.Generator("cuda").manual_seed(5)
    y = torch.randint(0, 9, (E,), generator=gen, **i32)
    y[torch.rand(E, generator=gen, device="cuda") < 0.4] = IGNORE
    y[:2 * 3001] = IGNORE      # rows in which nothing counts
    row_off, tile_off = np.concatenate([[0], np.cumsum(rows)]), np.concatenate([[0], np.cumsum(size)])
    tiles = odb.Tiles(torch.tensor(rows, **i32), torch.tensor(cols, **i32), torch.from_numpy(row_off).cuda(),
                      torch.from_numpy(tile_off).cuda(), y, R)
    t = torch.log(torch.rand(E, 1, generator=gen, device="cuda") * 0.9 + 0.05)
    s = torch.log(torch.rand(E, 1, generator=gen, device="cuda") * 0.9 + 0.05)
    ws = torch.full((odb.odb_distill_workspace_size(tiles, 1),), 0xa5, dtype=torch.uint8, device="cuda")
    loss, mean, grad = torch.empty(K, device="cuda"), torch.empty(K, device="cuda"), torch.full((E, 1), 7.0, device="cuda")
    count, status = torch.empty(K, **i64), torch.zeros(1, **i32)
    for _ in range(2):
        odb.odb_distill_loss(tiles, odb.DistillParams(reduce=reduce), s, t, loss, mean, count, ws, grad_student=grad,
                             status=status)
    assert int(status.item()) == 0
    p = t[:, 0].double().exp()
    D = p * (t[:, 0].double() - s[:, 0].double())
    for k in range(K):
        a, b = tile_off[k], tile_off[k + 1]
        if a == b:
            assert int(count[k]) == 0 and float(mean[k]) == 0
            continue
        on = (y[a:b] != IGNORE).view(rows[k], cols[k])
        on[:, 0] = False
        n = int(on.sum())
        assert int(count[k]) == n
        if reduce == 0:
            f = on.double() / max(n, 1)
        else:
            per = on.sum(1, keepdim=True)
            f = on.double() / per.clamp(min=1) / (per > 0).sum().clamp(min=1)
        f = f.view(-1)
        # a term costs about 10 roundings (a logarithm of 3, a power of 3, products), sums are in 64 bits
        want, size_of = float((f * D[a:b]).sum()), float((f * D[a:b].abs()).sum())
        assert abs(float(mean[k]) - want) <= 16 * U * size_of + 2 * U * abs(want), k
        want = -(f * p[a:b])
        assert bool(((grad[a:b, 0].double() - want).abs() <= 16 * U * want.abs()).all()), k
