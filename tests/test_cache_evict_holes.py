"""Eviction where the block table lacks pages: all that a call writes, against
the oracle, on every path of the selection."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests.cache_util import clone, get, same_bits
from tests.test_gpu_cache_evict import filled


def test_oracle_by_hand():
    w, order = [5.0, 0.0, 3.0, 3.0, 1.0, 4.0], [0, 1, 2, 3, 4, 5]
    hole = lambda *gone: [i not in gone for i in range(6)]
    assert oc.evict(w, order, 6, 3, 0, hole()) == oc.evict(w, order, 6, 3, 0)
    assert oc.evict(w, order, 6, 3, 0, hole(1)) == [0, -1, 5]       # two have room: 5.0 and 4.0
    assert oc.evict(w, order, 6, 3, 0, hole(0)) == [-1, 5, 2]       # of two of 3.0 the lower slot
    assert oc.evict(w, order, 6, 3, 0, hole(5)) == [0, 3, 2]        # a token that is not there does not count
    assert oc.evict(w, order, 6, 3, 2, hole(0, 1)) == [-1, -1, 4]   # of the latest the lower slot
    assert oc.evict(w, order, 6, 3, 0, hole(0, 1, 2)) == [-1, -1, -1]
    assert oc.evict(w, order, 6, 6, 0, hole(1, 5)) == [0, -1, 2, 3, 4, -1]


def check(old, whole, c, there, budget, recent, kept, state, weights, order, apart):
    """``old``: the cache before, ``whole``: the same with all its pages."""
    KV, page = c.k.shape[1], c.k.shape[2]
    held, seen = old.state.tolist()
    want, new_w, new_o = clone(old), None, None
    new_w = torch.full_like(old.weights, -1.0) if apart else want.weights
    new_o = torch.full_like(old.order, -1) if apart else want.order
    for b, n in enumerate(held):
        w, o = get(whole, "weights", b, n), get(whole, "order", b, n)
        for h in range(KV):
            src = oc.evict(w[h], o[h], seen[b], budget, recent, there[b][:n])
            assert kept[b, h].tolist() == src + [-1] * (budget - len(src)), (b, h)
            d = torch.tensor([i for i, s in enumerate(src) if s >= 0], device="cuda", dtype=torch.int64)
            s = torch.tensor([s for s in src if s >= 0], device="cuda", dtype=torch.int64)
            sp, so = whole.block_table[b].long()[s // page], s % page
            dp, do = whole.block_table[b].long()[d // page], d % page
            for name in ("k", "v"):
                getattr(want, name)[dp, h, do] = getattr(whole, name)[sp, h, so]
            new_w[dp, h, do], new_o[dp, h, do] = whole.weights[sp, h, so], whole.order[sp, h, so]
        want.state[0, b] = min(n, budget)
    assert torch.equal(state, want.state)
    assert same_bits(c.k, want.k) and same_bits(c.v, want.v)
    assert same_bits(weights, new_w) and torch.equal(order, new_o)


# (lengths, budget, recent, page): few evictions, one workgroup of each size, chunks with many and with a few
CASES = (((70, 66, 64, 40), 64, 9, 16), ((400, 401, 90), 100, 40, 32), ((3000, 2051, 2050), 2048, 300, 64),
         ((8100, 5000), 1000, 999, 16), ((20000, 9001, 300), 9000, 700, 128), ((30011, 16500), 8192, 100, 64))


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,budget,recent,page", CASES, ids=lambda v: str(v).replace(" ", ""))
@pytest.mark.parametrize("weights", ("random", "equal", "odd"))
@pytest.mark.parametrize("gone", ("below", "beyond", "both", "all below", "most"))
def test_missing_pages(lengths, budget, recent, page, weights, gone):
    whole = filled(lengths, 2, 8, page, "bf16", 5, weights=weights)
    c = clone(whole)
    r = np.random.default_rng(7)
    edge, blocks = budget // page, c.block_table.shape[1]
    there = []
    for b in range(len(lengths)):
        share = {"below": (0.3, 0.0), "beyond": (0.0, 0.4), "both": (0.2, 0.3), "all below": (1.0, 0.1),
                 "most": (0.9, 0.9)}[gone]
        out = r.random(blocks) < np.where(np.arange(blocks) < edge, share[0], share[1])
        if gone == "all below":
            out[: -(-budget // page)] = True
        for i, j in enumerate(np.flatnonzero(out)):
            c.block_table[b, int(j)] = (-1, c.k.shape[0], 2 ** 31 - 1, -(2 ** 31))[i % 4]
        there.append(np.repeat(~out, page))
    before = clone(c)
    for apart in (True, False):                     # the second call changes the cache
        kept = torch.full((len(lengths), 2, budget), -9, dtype=torch.int32, device="cuda")
        new = dict(new_state=torch.zeros_like(c.state), new_weights=torch.full_like(c.weights, -1.0),
                   new_order=torch.full_like(c.order, -1)) if apart else {}
        old = clone(before)
        own = clone(before)
        m.mosaic_cache_evict(own, budget, recent, kept=kept, **new)
        check(old, whole, own, there, budget, recent, kept, new.get("new_state", own.state),
              new.get("new_weights", own.weights), new.get("new_order", own.order), apart)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,budget", (((64, 10), 64), ((9000, 20), 9000)))
def test_nothing_to_evict(lengths, budget):
    """Within the budget every token stays; kept tells which slots hold one."""
    c = filled(lengths, 2, 8, 16, "f32", 15)
    c.block_table[0, 1], c.block_table[1, 0] = -1, c.k.shape[0]
    old = clone(c)
    kept = torch.full((2, 2, budget), -9, dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, budget, 3, kept=kept)
    for b, (n, lo) in enumerate(zip(lengths, (16, 0))):
        want = torch.arange(budget, dtype=torch.int32, device="cuda")
        want[lo: lo + 16] = -1
        want[n:] = -1
        assert (kept[b] == want).all()
    assert torch.equal(c.state, old.state) and same_bits(c.weights, old.weights) and same_bits(c.k, old.k)
