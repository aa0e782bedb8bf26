"""The gradient of lists, the same bit for bit from call to call."""
import pytest

from _losses import IGNORE

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


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
