"""Eviction by accumulated weight against the oracle: whole numbers and bits that
are moved, so every comparison is exact."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests.cache_util import DT, clone, get, make_cache, put, same_bits, seeded

pytestmark = pytest.mark.gpu


def filled(lengths, kv, dim, page, cache, seed, layout="heads", weights="random", shuffled=True):
    """A cache whose sequences have evicted before (order out of order, some tokens gone)."""
    seen = [n + 3 * b for b, n in enumerate(lengths)]
    c = make_cache(lengths, kv, dim, page, cache, seed, layout=layout, evicts=True, seen=seen)
    r = np.random.default_rng(seed)
    for b, n in enumerate(lengths):
        order = np.stack([np.sort(r.choice(seen[b], n, replace=False)) for _ in range(kv)]) if n else np.zeros((kv, 0), int)
        w = r.exponential(size=(kv, n)).astype(np.float32)
        if weights == "ties":
            w = np.round(w * 2) / 2
        elif weights == "equal":
            w[:] = 0.25
        elif weights == "odd":
            w = r.choice([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-40, -1e-40, 3.0, -2.0, 1e38, np.finfo(np.float32).min,
                          np.finfo(np.float32).max], size=(kv, n)).astype(np.float32)
        if shuffled:
            for h in range(kv):
                order[h, : n // 2] = r.permutation(order[h, : n // 2])
        put(c, "weights", b, torch.from_numpy(w).cuda())
        put(c, "order", b, torch.from_numpy(order.astype(np.int32)).cuda())
    return c


def check(c, old, budget, recent, kept=None, max_len=None, state=None, weights=None, order=None):
    KV, page = c.k.shape[1], c.k.shape[2]
    held, seen = old.state.tolist()
    want = clone(old)
    nw = want.weights if weights is None else torch.full_like(old.weights, -1.0)
    no = want.order if order is None else torch.full_like(old.order, -1)
    for b, n in enumerate(held):
        n = max(0, min(n, c.slots if max_len is None else max_len))
        w, o = get(old, "weights", b, n), get(old, "order", b, n)
        for h in range(KV):
            src = oc.evict(w[h], o[h], seen[b], budget, recent)
            if kept is not None:
                assert kept[b, h].tolist() == src + [-1] * (budget - len(src)), (b, h)
            s, d = torch.tensor(src, device="cuda", dtype=torch.int64), torch.arange(len(src), device="cuda")
            sp, so = old.block_table[b].long()[s // page], s % page
            dp, do = old.block_table[b].long()[d // page], d % page
            for name in ("k", "v"):
                getattr(want, name)[dp, h, do] = getattr(old, name)[sp, h, so]
            nw[dp, h, do], no[dp, h, do] = old.weights[sp, h, so], old.order[sp, h, so]
        want.state[0, b] = min(n, budget)
    assert torch.equal(c.state if state is None else state, want.state)
    assert same_bits(c.k, want.k) and same_bits(c.v, want.v)
    assert same_bits(c.weights if weights is None else weights, nw)
    assert torch.equal(c.order if order is None else order, no)


@pytest.mark.parametrize("cache", tuple(DT))
@pytest.mark.parametrize("lengths,budget,recent", (
    ((1, 2, 3), 1, 0), ((1, 2, 3), 1, 1), ((0, 5, 64, 65), 64, 10), ((17, 33, 100), 16, 16), ((300, 7, 301), 300, 0),
    ((1000, 999), 37, 5), ((129, 2500), 1023, 200), ((40, 41), 100, 3)))
def test_evict(cache, lengths, budget, recent):
    for dim, page, layout in ((64, 16, "heads"), (80, 64, "tokens")):
        c = filled(lengths, 2, dim, page, cache, 5, layout)
        old = clone(c)
        kept = torch.full((len(lengths), 2, budget), -9, dtype=torch.int32, device="cuda")
        m.mosaic_cache_evict(c, budget, recent, kept=kept)
        check(c, old, budget, recent, kept)


@pytest.mark.parametrize("weights", ("ties", "equal", "odd"))
@pytest.mark.parametrize("budget", (1, 100, 1500, 4999))
def test_ties_and_odd_numbers(weights, budget):
    """Ties to the lowest slot; infinities, zeros of both signs, NaN."""
    c = filled((5000, 1200), 3, 8, 32, "f16", 15, weights=weights)
    old = clone(c)
    kept = torch.empty((2, 3, budget), dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, budget, budget // 3, kept=kept)
    check(c, old, budget, budget // 3, kept)


@pytest.mark.parametrize("kv,dim,cache", ((1, 256, "f32"), (8, 128, "bf16")))
def test_long(kv, dim, cache):
    """More slots than one workgroup takes at a time, more than one round of them."""
    c = filled((70001, 9000), kv, dim, 128, cache, 25, weights="ties")
    old = clone(c)
    kept = torch.empty((2, kv, 33333), dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, 33333, 1111, kept=kept)
    check(c, old, 33333, 1111, kept)


@pytest.mark.parametrize("slots", (1024, 1040, 4096, 4112, 8192, 8208, 16400))
@pytest.mark.parametrize("fewer", (1, 4, 5, 600))
def test_where_the_kernels_change(slots, fewer):
    """A full table of as many slots as one workgroup takes and one page more,
    with few and many evictions; other sequences are shorter, one stays whole."""
    lengths = (slots, slots - fewer, slots - fewer + 1, 700, slots - 1)
    c = filled(lengths, 2, 8, 16, "bf16", 27, weights="ties")
    budget = slots - fewer
    for apart in (False, True):
        old = clone(c)
        kept = torch.full((5, 2, budget), -9, dtype=torch.int32, device="cuda")
        new = dict(new_state=torch.zeros_like(c.state), new_weights=torch.full_like(c.weights, -1.0),
                   new_order=torch.full_like(c.order, -1)) if apart else {}
        m.mosaic_cache_evict(c, budget, 3, kept=kept, **new)
        check(c, old, budget, 3, kept, state=new.get("new_state"), weights=new.get("new_weights"),
              order=new.get("new_order"))
        c = old


def test_no_pages():
    """A pool without pages: nothing is there to evict, lengths are cut."""
    empty = torch.empty((0, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    numbers = torch.empty((0, 2, 16), device="cuda")
    c = m.KVCache(empty, empty, torch.full((2, 3), -1, dtype=torch.int32, device="cuda"),
                  torch.tensor([[40, 5], [40, 5]], dtype=torch.int32, device="cuda"), numbers, numbers.int())
    m.mosaic_cache_evict(c, 20, 3)
    assert c.state.tolist() == [[20, 5], [40, 5]]
    q = torch.ones((2, 256), device="cuda")
    out = torch.ones_like(q)
    m.mosaic_cache_attend(c, q, 4, out)
    assert not out.any()
    m.mosaic_cache_append(c, torch.ones((2, 512), device="cuda"), 4, out)
    assert c.state.tolist() == [[21, 6], [41, 6]] and torch.equal(out, q)


def test_apart():
    """State, weights and order written elsewhere: the same call can be made
    again with the same result."""
    c = filled((500, 90, 3), 2, 64, 16, "bf16", 35)
    old = clone(c)
    for _ in range(2):
        state, w, o = torch.full_like(c.state, -1), torch.full_like(c.weights, -1.0), torch.full_like(c.order, -1)
        kept = torch.empty((3, 2, 100), dtype=torch.int32, device="cuda")
        m.mosaic_cache_evict(c, 100, 20, max_len=500, new_state=state, new_weights=w, new_order=o, kept=kept)
        check(c, old, 100, 20, kept, state=state, weights=w, order=o)
        assert same_bits(c.weights, old.weights) and torch.equal(c.order, old.order)
        assert torch.equal(c.state, old.state)


def test_lengths_are_bounded():
    c = filled((200, 200, 200), 2, 64, 16, "bf16", 45)
    c.state[0] = torch.tensor([-4, 1 << 30, 130], dtype=torch.int32, device="cuda")
    old = clone(c)
    m.mosaic_cache_evict(c, 50, 10)
    check(c, old, 50, 10)
    c = clone(old)
    m.mosaic_cache_evict(c, 50, 10, max_len=120)
    check(c, old, 50, 10, max_len=120)
    c = clone(old)
    m.mosaic_cache_evict(c, 50, 10, max_len=0)
    assert c.state[0].tolist() == [0, 0, 0] and same_bits(c.k, old.k)


def test_pages_that_are_not_there():
    """Tokens of missing pages go first; nothing is written outside the pool."""
    c = filled((160, 160), 2, 64, 16, "bf16", 55)
    c.block_table[0, 2], c.block_table[1, 9], c.block_table[1, 1] = -1, c.k.shape[0], 2 ** 31 - 1
    old = clone(c)
    kept = torch.full((2, 2, 64), -9, dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, 64, 0, kept=kept)
    used = set()
    for b, gone in ((0, {2}), (1, {1, 9})):
        for h in range(2):
            src = kept[b, h].tolist()
            assert all(s // 16 not in gone for i, s in enumerate(src) if s >= 0 and i // 16 not in gone)
            for i, s in enumerate(src):
                if i // 16 in gone or s < 0:
                    continue
                p, f = int(c.block_table[b, i // 16]), int(c.block_table[b, s // 16])
                assert same_bits(c.k[p, h, i % 16], old.k[f, h, s % 16])
                assert same_bits(c.v[p, h, i % 16], old.v[f, h, s % 16])
                used.add(p)
    rest = [p for p in range(c.k.shape[0]) if p not in used]
    assert same_bits(c.k[rest], old.k[rest]) and same_bits(c.weights[rest], old.weights[rest])


def test_steps_in_a_graph():
    """A decode loop at its budget: append and evict captured together, every
    replay against the eager calls."""
    big = make_cache((20, 32), 2, 64, 16, "bf16", 66, room=4, evicts=True)
    want = clone(big)
    x = torch.randn((2, 8 * 64), generator=seeded(67), device="cuda")
    q = torch.empty((2, 256), device="cuda")
    def step(cache):
        m.mosaic_cache_append(cache, x, 4, q)
        m.mosaic_cache_attend(cache, q, 4, q2, accumulate=True)
        m.mosaic_cache_evict(cache, 24, 4)
    q2 = torch.empty_like(q)
    step(big), step(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(big)
    for i in range(12):
        x.copy_(torch.randn((2, 8 * 64), generator=seeded(70 + i), device="cuda"))
        graph.replay()
        out = q2.clone()
        step(want)
        torch.cuda.synchronize()
        assert torch.equal(out, q2) and torch.equal(big.state, want.state)
        for name in ("k", "v", "weights", "order"):
            assert same_bits(getattr(big, name), getattr(want, name)), (i, name)
    assert want.state[0].tolist() == [24, 24]


def test_far_pages():
    """Rows whose offsets pass 32 bits."""
    pages = 1 << 15
    small = filled((200,), 8, 128, 64, "bf16", 75)
    old = clone(small)
    far = torch.tensor([pages - 1, 5, pages - 2, 16385], device="cuda")
    src = small.block_table[0].long()
    pool = [torch.empty((pages, 8, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]      # 4.3 GB each
    w = torch.zeros((pages, 8, 64), device="cuda")
    o = torch.zeros((pages, 8, 64), dtype=torch.int32, device="cuda")
    pool[0][far], pool[1][far], w[far], o[far] = small.k[src], small.v[src], small.weights[src], small.order[src]
    big = m.KVCache(pool[0], pool[1], far.to(torch.int32)[None, :], small.state.clone(), w, o)
    m.mosaic_cache_evict(small, 70, 9)
    m.mosaic_cache_evict(big, 70, 9)
    for name in ("k", "v", "weights", "order"):
        assert same_bits(get_rows(big, name), get_rows(small, name))
    check(small, old, 70, 9)


def get_rows(c, name):
    return getattr(c, name)[c.block_table[0].long()]


def test_refusals():
    c = filled((40,), 2, 64, 16, "bf16", 85)
    m.mosaic_cache_evict(clone(c), 10, 2)
    for bad in ((0, 0, {}), (-1, 0, {}), (10, 11, {}), (10, -1, {}), (10, 2, dict(max_len=-1))):
        with pytest.raises(m.MosaicError) as e:
            m.mosaic_cache_evict(c, bad[0], bad[1], **bad[2])
        assert e.value.status == m.STATUS_INVALID_ARG
    P = c.weights.numel()
    flat = torch.zeros(P + 64, device="cuda")
    half = m.KVCache(c.k, c.v, c.block_table, c.state, flat[:P].view_as(c.weights), c.order)
    with pytest.raises(m.MosaicError):                      # new_weights half over weights
        m.mosaic_cache_evict(half, 10, 2, new_weights=flat[64:].view_as(c.weights))
    for bad in (dict(kept=torch.zeros((1, 2, 9), dtype=torch.int32, device="cuda")),
                dict(kept=torch.zeros((1, 2, 10), dtype=torch.int64, device="cuda")),
                dict(new_state=c.state.long()), dict(new_weights=c.weights[:1]), dict(new_order=c.weights)):
        with pytest.raises(ValueError):
            m.mosaic_cache_evict(c, 10, 2, **bad)
    with pytest.raises(ValueError):
        m.mosaic_cache_evict(m.KVCache(c.k, c.v, c.block_table, c.state, c.weights), 10, 2)
