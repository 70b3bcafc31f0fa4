"""The sort of many pairs to many experts against a stable sort, on the device."""
import pytest
import torch

from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,k,E", [(1 << 20, 1, 1024), (1 << 17, 8, 1000), (40_001, 32, 256), (3_000_001, 1, 3)])
def test_against_a_stable_sort(cuda_device, T, k, E):
    gen = torch.Generator(device="cuda").manual_seed(T)
    # popular and unpopular experts, one pair in fifty over capacity
    ids = (torch.rand(T, k, device="cuda", generator=gen).square() * E).int().clamp(max=E - 1)
    ids[torch.rand(T, k, device="cuda", generator=gen) < 0.02] = -1
    r = layers.route(ids, E)
    key = torch.where(ids < 0, E, ids).reshape(-1)
    order = torch.argsort(key, stable=True)
    used = int((key < E).sum())
    slot = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    slot[order[:used]] = torch.arange(used, dtype=torch.int32, device="cuda")
    source = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    source[:used] = order[:used].int()
    counts = torch.bincount(key, minlength=E + 1)[:E]
    assert torch.equal(r.offsets, torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int())
    assert torch.equal(r.slot.reshape(-1), slot) and torch.equal(r.source, source)
