"""Which positions are split over blocks: those whose parts are fewer rounds of loads than the chip's blocks would be
shared by (without a GPU: what is split needs a workspace)."""
import ctypes

import pytest

import paper_2606_19989_amd as odb
from test_losses_host import _logits


@pytest.mark.parametrize("n,V,k,split", [
    (1, 151936, 20, True), (48, 151936, 20, True), (128, 151936, 64, True), (1, 50000, 20, True), (1, 49152, 20, False),
    (64, 50000, 20, False), (128, 50000, 64, False), (256, 151936, 20, False), (512, 50000, 20, False),
    (512, 151936, 64, False), (512, 250000, 20, False), (128, 50000, 128, True), (512, 50000, 128, False),
    (512, 151936, 128, True), (513, 1000000, 20, False),
])
def test_split_positions(n, V, k, split):
    x = _logits(dtype=odb.ODB_BFLOAT16, rows=1, cols=n, vocab=V, row_stride=n * V, col_stride=V)
    assert (odb.load().odb_token_top_workspace_size(ctypes.byref(x), k) > 256) == split
