"""Attention of one new token over a paged cache in 4 bits, against the float64
oracle on the values that the codes stand for.

Tolerance as in test_gpu_cache_attend.py (an output by (2 (dim + 4) S + n + 16)
u A from float32 scores, weights and sums, S the largest sum of |q k| scale and
A = sum p |v|), and 2^-17 of a weight where two bf16 parts of it are multiplied
(16-bit activations; three hold all 24 bits). A float32 query is three bf16
parts (all of it), an f16 one two. The output is rounded once."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests import e2m1_util as eu
from tests.cache_util import DT, TINY, UNIT, f64, same_bits, seeded

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PARTS = {"f32": 0.0, "bf16": 2.0 ** -17, "f16": 2.0 ** -17}


def check(c, q, heads, out, act, scale, before=None, holes=(), max_len=None):
    KV, page, D = c.k.shape[1], c.k.shape[2], c.head_dim
    G = heads // KV
    got, qs = f64(out).reshape(-1, heads, D), f64(q).reshape(-1, heads, D)
    for b, n in enumerate(c.state[0].tolist()):
        n = max(0, min(n, c.slots if max_len is None else max_len))
        there = np.ones(n, dtype=bool)
        for s, j in holes:
            if s == b:
                there[j * page: (j + 1) * page] = False
        if n == 0 or not there.any():
            assert not got[b].any()
            continue
        k, v = eu.get(c, "k", b, n)[:, there], eu.get(c, "v", b, n)[:, there]
        for h in range(KV):
            o, p = oc.attend(qs[b, h * G: (h + 1) * G], k[h], v[h], scale)
            S = abs(scale) * (np.abs(qs[b, h * G: (h + 1) * G]) @ np.abs(k[h]).T).max(axis=1, keepdims=True)
            A = p @ np.abs(v[h])
            rel = (2 * (D + 4) * S + n + 16) * U
            off = (rel + PARTS[act]) * A
            tol = off + UNIT[act] * (np.abs(o) + off) + TINY[act]
            err = np.abs(got[b, h * G: (h + 1) * G] - o)
            assert (err <= tol).all(), (b, h, err.max(), tol[err > tol][:3])
            if before is not None:
                want = before[b][h][there] + p.sum(axis=0)
                now = eu.get(c, "weights", b, n)[h][there]
                assert (np.abs(now - want) <= (rel * p).sum(axis=0) + 4 * U * want + 1e-38).all()


def run(c, heads, act, seed, accumulate=False, scale=None, std=1.0, **kw):
    D = c.head_dim
    q = (torch.randn((c.batch, heads * D), generator=seeded(seed), device="cuda") * std).to(DT[act])
    out = torch.full_like(q, float("nan"))
    m.mosaic_cache_attend(c, q, heads, out, scale=scale, accumulate=accumulate, **kw)
    return q, out, 1.0 / math.sqrt(D) if scale is None else scale


LENGTHS = ((1,), (0, 1, 2, 15, 16, 17, 31, 32, 33), (63, 64, 65, 127, 129, 0, 300), (2047, 1025))
# (heads, kv_heads, dim): padded head dimensions, partial quarters of a row, one and several blocks of heads
SHAPES = ((4, 2, 64), (8, 1, 128), (6, 6, 128), (6, 2, 80), (10, 2, 8), (33, 1, 64), (3, 3, 256), (14, 2, 104),
          (5, 1, 40), (4, 1, 72), (4, 2, 136), (2, 1, 200), (16, 1, 16), (8, 2, 96), (4, 4, 232))


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim", SHAPES)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: f"len{max(v)}")
def test_attend(act, heads, kv, dim, lengths):
    c = eu.make_cache(lengths, kv, dim, 16 if max(lengths) < 100 else 64, 11, layout="tokens" if dim in (80, 136) else "heads",
                      gap=16 if dim == 104 else 0)
    q, out, scale = run(c, heads, act, 12)
    check(c, q, heads, out, act, scale)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim", ((4, 2, 64), (8, 1, 128), (40, 2, 80), (3, 3, 256)))
@pytest.mark.parametrize("page", (16, 32, 128))
def test_weights_add_up(act, heads, kv, dim, page):
    """Two steps in a row; weights of other slots and the cache stay as they are."""
    lengths = (0, 1, 77, 513)
    c = eu.make_cache(lengths, kv, dim, page, 21, evicts=True, layout="tokens" if page == 32 else "heads")
    for step in range(2):
        old = eu.clone(c)
        before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)]
        q, out, scale = run(c, heads, act, 22 + step, accumulate=True)
        check(c, q, heads, out, act, scale, before)
        used = torch.zeros_like(c.weights, dtype=torch.bool)
        for b, n in enumerate(lengths):
            p, o = eu.where(c, b, 0, n)
            used[p, :, o] = True
        assert same_bits(c.weights[~used], old.weights[~used])
        assert torch.equal(c.k, old.k) and torch.equal(c.v, old.v) and torch.equal(c.state, old.state)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim", ((71, 1, 64), (40, 1, 128), (34, 2, 128), (20, 1, 256), (33, 1, 24)))
def test_many_query_heads_per_key_head(act, heads, kv, dim):
    lengths = (130, 0, 1, 700)
    c = eu.make_cache(lengths, kv, dim, 32, 25, evicts=True)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)]
    q, out, scale = run(c, heads, act, 26, accumulate=True)
    check(c, q, heads, out, act, scale, before)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("batch", (64, 65, 200))
def test_many_sequences(act, batch):
    """More sequences than a wave has lanes, most of them short, many empty."""
    r = np.random.default_rng(batch)
    lengths = [int(n) if r.random() < 0.6 else 0 for n in r.exponential(60, batch)]
    lengths[0], lengths[-1], lengths[batch // 2] = 0, 0, 1500
    c = eu.make_cache(lengths, 2, 64, 16, 27, evicts=True)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)]
    q, out, scale = run(c, 6, act, 28, accumulate=True)
    check(c, q, 6, out, act, scale, before)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim,longest", ((80, 1, 64, 12001), (150, 3, 32, 9000), (24, 12, 64, 3000),
                                                  (71, 71, 16, 1100), (300, 300, 8, 700), (1024, 1024, 8, 260),
                                                  (96, 2, 256, 4500)))
def test_shares(act, heads, kv, dim, longest):
    """Head counts whose shares do not divide the chip."""
    lengths = (longest, 0, 300 if kv < 300 else 20)
    c = eu.make_cache(lengths, kv, dim, 64, 41, evicts=True, layout="tokens" if kv == 12 else "heads")
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)]
    q, out, scale = run(c, heads, act, 42, accumulate=True)
    check(c, q, heads, out, act, scale, before)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("std", (0.0, 0.01, 40.0))
def test_flat_and_sharp(act, std):
    """All weights alike, and one that takes all of it."""
    c = eu.make_cache((300, 4100), 2, 128, 64, 31)
    q, out, scale = run(c, 8, act, 32, std=std)
    check(c, q, 8, out, act, scale)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("spread", (2.0 ** -100, 2.0 ** 60))
def test_scales_far_from_one(act, spread):
    """Keys a hundred powers of two down or sixty up, scores brought back by
    ``scale``; values as far where the outputs' type reaches."""
    c = eu.make_cache((70,), 2, 64, 16, 33, scale=spread)
    assert abs(np.log2(np.abs(eu.get(c, "k", 0, 70)).max() / spread)) < 4
    if act == "f16":
        eu.put(c, "v", 0, torch.randn((2, 70, 64), generator=seeded(3), device="cuda"))
    q, out, scale = run(c, 4, act, 34, scale=0.125 / spread)
    check(c, q, 4, out, act, scale)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("scale", (0.0, -0.2, 1.5))
def test_scale(act, scale):
    """Zero weighs all tokens alike, a negative one turns the scores round."""
    c = eu.make_cache((77, 1, 0, 300), 2, 64, 16, 43, evicts=True)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate((77, 1, 0, 300))]
    q, out, _ = run(c, 4, act, 44, accumulate=True, scale=scale)
    check(c, q, 4, out, act, scale, before)


@pytest.mark.parametrize("act", eu.ACTS)
def test_max_len_and_lengths_out_of_range(act):
    c = eu.make_cache((200, 33, 64, 64), 2, 64, 32, 35)
    q, out, scale = run(c, 4, act, 36, max_len=50)
    check(c, q, 4, out, act, scale, max_len=50)
    c.state[0, 1], c.state[0, 2] = -5, 10 ** 6
    c.block_table[2, 2:] = -1
    q, out, scale = run(c, 4, act, 37)
    got = f64(out)
    assert not got[1].any()
    c.state[0, 2] = 64
    q2, out2, _ = run(c, 4, act, 37)
    assert torch.equal(out[2], out2[2])


@pytest.mark.parametrize("act", eu.ACTS)
def test_pages_that_are_not_there(act):
    c = eu.make_cache((200, 33, 64), 2, 64, 32, 38, evicts=True)
    c.block_table[0, 0], c.block_table[0, 3], c.block_table[2, 0], c.block_table[2, 1] = -1, c.k.shape[0], -7, 2 ** 31 - 1
    saved = c.block_table.clone()
    c.block_table.clamp_(0, c.k.shape[0] - 1)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate((200, 33, 64))]
    c.block_table.copy_(saved)
    q, out, scale = run(c, 4, act, 39, accumulate=True)
    c.block_table.clamp_(0, c.k.shape[0] - 1)
    check(c, q, 4, out, act, scale, before, holes=((0, 0), (0, 3), (2, 0), (2, 1)))


@pytest.mark.parametrize("act", eu.ACTS)
def test_nan_and_infinities(act):
    """NaN among the keys or values reaches what they weigh on and nothing else; an
    infinite query gives what the formulas give."""
    c = eu.make_cache((90, 40), 2, 64, 16, 51)
    clean = eu.clone(c)
    p, o = eu.where(c, 0, 70, 1)
    c.k[p, 0, o, 32 + 3] = 255                          # elements 24 to 31 of a key of head 0
    p, o = eu.where(c, 1, 5, 1)
    c.v[p, 1, o, 32 + 2] = 255                          # elements 16 to 23 of a value of head 1
    q, out, scale = run(c, 4, act, 52)
    _, want, _ = run(clean, 4, act, 52)
    got = out.view(2, 4, 64)
    bad = torch.isnan(got)
    expect = torch.zeros_like(bad)
    expect[0, :2] = True
    expect[1, 2:, 16: 24] = True
    assert torch.equal(bad, expect) and torch.equal(got[~bad], want.view(2, 4, 64)[~bad])
    q[0, 3], q[1, 200] = float("inf"), float("nan")
    out = torch.empty_like(q)
    m.mosaic_cache_attend(clean, q, 4, out)
    got = f64(out).reshape(2, 4, 64)
    for b, n in ((0, 90), (1, 40)):
        for g in range(4):
            with np.errstate(all="ignore"):
                o, _ = oc.attend(f64(q)[b].reshape(4, 64)[g: g + 1], eu.get(clean, "k", b, n)[g // 2], eu.get(clean, "v", b, n)[g // 2], scale)
            assert np.array_equal(np.isnan(got[b, g]), np.isnan(o[0]))


def test_scores_of_minus_infinity():
    """An infinite query element on keys of one sign there: scores of -inf are no
    weight, and a row of nothing else gives zeros."""
    c = eu.make_cache((40, 40), 1, 16, 16, 53)
    for b in range(2):
        k = torch.randn((1, 40, 16), generator=seeded(54 + b), device="cuda")
        k[:, :, 0] = -1.0 - k[:, :, 0].abs()
        if b == 0:
            k[:, 7, 0] = 0.0                            # NaN: infinity times nothing
        eu.put(c, "k", b, k)
    for act in eu.ACTS:
        q = torch.randn((2, 16), generator=seeded(55), device="cuda").to(DT[act])
        q[:, 0] = float("inf")
        out = torch.empty_like(q)
        m.mosaic_cache_attend(c, q, 1, out)
        assert torch.isnan(out[0]).all() and not out[1].any()


@pytest.mark.parametrize("act", ("f32", "bf16"))
def test_largest_queries(act):
    """Elements at the end of the type's range, which bf16 rounds to infinity, on
    keys that bring the scores back."""
    c = eu.make_cache((50,), 1, 16, 16, 56, scale=2.0 ** -126)
    q = torch.randn((1, 16), generator=seeded(57), device="cuda").sign() * torch.finfo(DT[act]).max
    q = q.to(DT[act])
    eu.put(c, "v", 0, torch.randn((1, 50, 16), generator=seeded(58), device="cuda"))
    out = torch.empty_like(q)
    m.mosaic_cache_attend(c, q, 1, out, scale=0.125)
    check(c, q, 1, out, act, 0.125)


def test_strided_rows():
    c = eu.make_cache((20, 77), 2, 64, 16, 61, gap=16)
    q, out, _ = run(c, 4, "f16", 62)
    wide_q = torch.zeros((2, 320), dtype=torch.float16, device="cuda")
    wide_o = torch.zeros((4, 328), dtype=torch.float16, device="cuda")
    wide_q[:, 8: 264] = q
    m.mosaic_cache_attend(c, wide_q[:, 8: 264], 4, wide_o[1:3, 16: 272])
    assert torch.equal(wide_o[1:3, 16: 272], out)
    wide_o[1:3, 16: 272] = 0
    assert not wide_o.any()


def test_shared_table():
    c = eu.make_cache((100,), 2, 64, 16, 63)
    shared = m.KVCache(c.k, c.v, c.block_table.expand(3, -1), torch.tensor([[100, 7, 64]] * 2, dtype=torch.int32, device="cuda"),
                       head_dim=64)
    q, out, scale = run(shared, 4, "f32", 64)
    check(shared, q, 4, out, "f32", scale)


@pytest.mark.parametrize("act", eu.ACTS)
def test_same_bits_every_time(act):
    c = eu.make_cache((3000, 10, 700, 0), 2, 128, 64, 65, evicts=True)
    first = None
    for _ in range(4):
        w = eu.clone(c)
        _, out, _ = run(w, 16, act, 66, accumulate=True)
        if first is None:
            first = (out, w.weights)
        assert torch.equal(out, first[0]) and same_bits(w.weights, first[1])


def test_side_stream_and_two_graphs():
    """Two captured graphs, each with its own workspace, replayed in turn with
    eager calls between them as the lengths grow."""
    c = eu.make_cache((100, 30), 2, 64, 16, 67, room=64)
    eu.put(c, "k", 0, torch.randn((2, 164, 64), generator=seeded(1), device="cuda"))
    eu.put(c, "v", 0, torch.randn((2, 164, 64), generator=seeded(2), device="cuda"))
    eu.put(c, "k", 1, torch.randn((2, 94, 64), generator=seeded(3), device="cuda"))
    eu.put(c, "v", 1, torch.randn((2, 94, 64), generator=seeded(4), device="cuda"))
    qs = [torch.randn((2, 256), generator=seeded(5 + i), device="cuda") for i in range(2)]
    outs = [torch.zeros((2, 256), device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.mosaic_cache_attend(c, qs[0], 4, outs[0])
    side.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.mosaic_cache_attend(c, qs[i], 4, outs[i])
        graphs.append(g)
    for step in range(4):
        c.state[0] += 16
        for i in (step % 2, 1 - step % 2):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
        for i in range(2):
            want = torch.empty_like(outs[i])
            m.mosaic_cache_attend(c, qs[i], 4, want)
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want)
            check(c, qs[i], 4, outs[i], "f32", 0.125)


def test_far_pages():
    """Rows more than 4 GiB into the cache."""
    dim, kv, page = 256, 8, 128
    width = m.KVCache.row_bytes(dim)
    pages = (9 << 29) // (kv * page * width)                    # 4.5 GiB
    k = torch.empty((pages, kv, page, width), dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    k[-4:], v[-4:] = 255, 255
    c = m.KVCache(k, v, torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device="cuda"),
                  torch.tensor([[200], [200]], dtype=torch.int32, device="cuda"), head_dim=dim)
    for i, name in enumerate(("k", "v")):
        eu.put(c, name, 0, torch.randn((kv, 200, dim), generator=seeded(70 + i), device="cuda"))
    q, out, scale = run(c, 16, "bf16", 72)
    check(c, q, 16, out, "bf16", scale)
    x, q2 = torch.randn((1, 32 * dim), generator=seeded(73), device="cuda"), torch.empty((1, 16 * dim), device="cuda")
    m.mosaic_cache_append(c, x, 16, q2)
    ko, vo = torch.empty((1, kv * dim), device="cuda"), torch.empty((1, kv * dim), device="cuda")
    m.mosaic_cache_read(c, ko, vo, first=torch.tensor([200], dtype=torch.int32, device="cuda"))
    want = oc.unpack_e2m1(oc.pack_e2m1(*oc.to_e2m1(f64(x)[:, 16 * dim:].reshape(2, kv, dim))), dim).reshape(2, kv * dim)
    assert np.array_equal(f64(ko)[0], want[0]) and np.array_equal(f64(vo)[0], want[1])


@pytest.mark.parametrize("layout", ("heads", "tokens"))
def test_evict_moves_rows(layout):
    """Eviction over 4 bits: survivors' rows move whole; attention over what is left."""
    lengths, budget, recent = (70, 10, 33), 32, 5
    c = eu.make_cache(lengths, 2, 80, 16, 81, layout=layout, evicts=True)
    old = eu.clone(c)
    kept = torch.empty((3, 2, budget), dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, budget, recent, kept=kept)
    for b, n in enumerate(lengths):
        left = min(n, budget)
        assert c.state[:, b].tolist() == [left, n]
        rows = {name: (eu.rows_of(c, name, b, 0, left), eu.rows_of(old, name, b, 0, n)) for name in ("k", "v")}
        for h in range(2):
            want = oc.evict(eu.get(old, "weights", b, n)[h], eu.get(old, "order", b, n)[h], n, budget, recent)
            assert kept[b, h, :left].tolist() == want[:left]
            for now, then in rows.values():
                assert np.array_equal(now[h], then[h][want[:left]])
            assert np.array_equal(eu.get(c, "weights", b, left)[h], eu.get(old, "weights", b, n)[h][want[:left]])
    q, out, scale = run(c, 4, "f32", 82)
    check(c, q, 4, out, "f32", scale)


def test_a_step_together():
    """Norms, positions, append, attention with weights and eviction, step by step
    in one graph, against the oracle on the cache before each step's eviction."""
    c = eu.make_cache((30, 31), 2, 64, 16, 91, room=8, evicts=True)
    x = torch.randn((2, 8 * 64), generator=seeded(92), device="cuda")
    q, out = torch.empty((2, 256), device="cuda"), torch.empty((2, 256), device="cuda")
    w = torch.rand(64, generator=seeded(93), device="cuda") + 0.5
    rotary, norm = m.Rotary(m.Rotary.frequencies(64, 32), [32]), m.QKNorm(w, w)

    def step(c):
        m.mosaic_cache_append_norm(c, x, 4, q, norm, rotary=rotary)
        m.mosaic_cache_attend(c, q, 4, out, accumulate=True)
        seen = eu.clone(c)
        m.mosaic_cache_evict(c, 32, 4)
        return seen
    eager = eu.clone(c)
    step(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.mosaic_cache_append_norm(c, x, 4, q, norm, rotary=rotary)
        m.mosaic_cache_attend(c, q, 4, out, accumulate=True)
        m.mosaic_cache_evict(c, 32, 4)
    eager = eu.clone(c)
    for i in range(5):
        x.copy_(torch.randn(x.shape, generator=seeded(95 + i), device="cuda"))
        graph.replay()
        got_q, got = q.clone(), out.clone()
        before = step(eager)
        assert torch.equal(q, got_q) and torch.equal(out, got)
        check(before, q, 4, out, "f32", 0.125)
        for name in ("state", "weights", "order", "k", "v"):
            assert same_bits(getattr(c, name), getattr(eager, name)), (i, name)


def test_refusals():
    c = eu.make_cache((3, 4), 2, 64, 16, 96)
    q, out = torch.zeros((2, 256), device="cuda"), torch.zeros((2, 256), device="cuda")
    m.mosaic_cache_attend(c, q, 4, out)
    for bad in (dict(heads=3), dict(heads=0), dict(scale=float("nan"))):
        with pytest.raises(m.MosaicError):
            m.mosaic_cache_attend(c, q, bad.get("heads", 4), out, scale=bad.get("scale"))
    for cache in (m.KVCache(c.k, c.v, c.block_table, c.state), m.KVCache(c.k, c.v, c.block_table, c.state, head_dim=128),
                  m.KVCache(c.k.view(torch.int8), c.v.view(torch.int8), c.block_table, c.state, head_dim=64)):
        with pytest.raises(ValueError):
            m.mosaic_cache_attend(cache, q, 4, out)
    with pytest.raises(m.MosaicError):                      # head_dim that the kernels do not take
        m.mosaic_cache_attend(m.KVCache(c.k, c.v, c.block_table, c.state, head_dim=60), q[:, :240], 4, out[:, :240])
    with pytest.raises(ValueError):
        m.mosaic_cache_attend(c, q.double(), 4, out.double())
    with pytest.raises(ValueError):
        m.mosaic_cache_attend(c, q, 4, out, accumulate=True)
