"""Eviction over tables of as many slots as the ABI takes, and of more moves
than one launch has workgroups for."""
import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests.cache_util import same_bits, seeded

pytestmark = pytest.mark.gpu


def test_most_slots():
    """2^30 slots, of which few are in use: the launches are sized by the table."""
    page, pages = 4096, 2
    k, v = (torch.randn((pages, 1, page, 8), generator=seeded(5), device="cuda").half() for _ in range(2))
    table = torch.full((1, 1 << 18), -1, dtype=torch.int32, device="cuda")
    table[0, :2] = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    state = torch.tensor([[5000], [6000]], dtype=torch.int32, device="cuda")
    weights = torch.rand((pages, 1, page), generator=seeded(6), device="cuda")
    order = torch.arange(pages * page, dtype=torch.int32, device="cuda").reshape(pages, 1, page)
    c = m.KVCache(k, v, table, state.clone(), weights.clone(), order.clone())
    assert c.slots == 1 << 30
    m.mosaic_cache_evict(c, 1 << 29, 7)
    assert torch.equal(c.state, state) and torch.equal(c.weights, weights) and torch.equal(c.order, order)
    # and with a budget that moves some
    want = m.KVCache(k.clone(), v.clone(), table[:, :2].contiguous(), state.clone(), weights.clone(), order.clone())
    m.mosaic_cache_evict(want, 4500, 7)
    m.mosaic_cache_evict(c, 4500, 7)
    for name in ("k", "v", "weights", "order", "state"):
        assert same_bits(getattr(c, name), getattr(want, name)), name


def test_many_moves():
    """Every token below the budget goes, every one beyond it moves."""
    budget, page = (1 << 20) + (1 << 19) + 77, 4096
    blocks = -(-2 * budget // page)
    k = torch.randint(0, 1 << 15, (blocks, 1, page, 8), generator=seeded(7), device="cuda", dtype=torch.int16).view(
        torch.bfloat16)
    v = k + 1
    table = torch.randperm(blocks, generator=seeded(8), device="cuda").to(torch.int32)[None]
    slot = torch.arange(blocks * page, device="cuda").reshape(blocks, 1, page)
    weights, order = torch.empty((blocks, 1, page), device="cuda"), torch.empty((blocks, 1, page), dtype=torch.int32, device="cuda")
    weights[table[0].long()] = (slot >= budget).float()
    order[table[0].long()] = slot.to(torch.int32)
    c = m.KVCache(k.clone(), v.clone(), table, torch.full((2, 1), 2 * budget, dtype=torch.int32, device="cuda"),
                  weights, order)
    kept = torch.full((1, 1, budget), -9, dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, budget, 0, kept=kept)
    assert torch.equal(kept[0, 0], torch.arange(budget, 2 * budget, dtype=torch.int32, device="cuda"))
    assert c.state.tolist() == [[budget], [2 * budget]]
    t = table[0].long()
    for name, old in (("k", k), ("v", v)):
        got = getattr(c, name)[t].reshape(-1, 8)[:budget]
        assert torch.equal(got.view(torch.int16), old[t].reshape(-1, 8)[budget: 2 * budget].contiguous().view(torch.int16))
    assert torch.equal(c.order[t].reshape(-1)[:budget], kept[0, 0]) and (c.weights[t].reshape(-1)[:budget] == 1).all()
