"""Routes of more tokens than a launch of two kernels takes: several chunks of tokens a thread of the scan, experts that are no multiple of
four, tokens that end inside a chunk.  Which experts, rows and slots is exact; ties go to the lower expert."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [(16385, 4, 2), (32768, 7, 3), (40000, 130, 8), (70001, 64, 6), (300007, 21, 2)])
def test_route(T, E, k):
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.randn(T, E, device="cuda", generator=g).bfloat16()
    x[5] = float("-inf")   # a token that takes no expert
    x[7, 1:] = float("nan")
    r = B.hlq_route(x, k)
    key = torch.nan_to_num(x.double(), nan=float("-inf"), neginf=float("-inf"))
    top, ids = torch.sort(key, dim=1, descending=True, stable=True)
    ids = torch.where(top[:, :k].isinf(), -1, ids[:, :k])
    assert torch.equal(r.ids.long(), ids)
    flat = ids.flatten()
    taken = torch.nonzero(flat >= 0).flatten()
    order = taken[torch.sort(flat[taken], stable=True).indices]
    n = order.numel()
    assert torch.equal(r.offsets.long(), torch.cat([torch.zeros(1, device="cuda").long(), torch.bincount(flat[taken], minlength=E).cumsum(0)]))
    assert torch.equal(r.rows[:n].long(), order // k) and bool((r.rows[n:] == -1).all())
    slots = torch.full((T * k,), -1, device="cuda")
    slots[order] = torch.arange(n, device="cuda")
    assert torch.equal(r.slots.flatten().long(), slots)
