"""New tokens with norms of queries and keys, into caches of 32, 16 and 4 bits.

In 16 and 32 bits against the float64 oracle. With u = 2^-24, the factor f is
rounded once, x f and (x f) w once each: 3 u of y; a turned element y c - z s
adds a rounding of each product and of the sum, 2 u (|y c| + |z s|) in all, on
5 u of these; one rounding more to the type it is stored in.

Every step is rounded by itself, so float32 arithmetic in that order gives the
same numbers, and a cache in 4 bits holds exactly the oracle's codes for them."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests import cache_util as cu
from tests import e2m1_util as eu
from tests.cache_util import DT, TINY, TYPES, UNIT, f64, same_bits, seeded

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 2.0 ** -20

# (sections, interleaved) by head dimension: whole heads, parts, several axes, ragged ends, nothing
ROTARY = {
    128: (((64,), False), ((16, 24, 24), False), ((64,), True), ((1,), False), ((24,), False), None),
    64: (((32,), False), ((5, 0, 7, 3), True), ((7, 6), False)),
    80: (((40,), False), ((20,), False), ((7, 13), True)),
    8: (((4,), False), ((1, 1, 1), True), ((3,), False)),
    16: (((8,), False),),
    24: (((8,), False), ((12,), True)),
    40: (((16,), False), None),
    256: (((128,), False), ((64, 64), True), ((100,), False)),
}
CASES = [(d, r) for d, rs in ROTARY.items() for r in rs]


def inputs(c, dim, heads, act, fresh, rot, seed, starts=True, text=False, norm=True, table_rows=300):
    KV = c.k.shape[1]
    rows = sum(fresh)
    g = seeded(seed)
    x = torch.randn((rows, (heads + 2 * KV) * dim), generator=g, device="cuda")
    x = (x * torch.randn((rows, 1), generator=g, device="cuda").exp()).to(DT[act])
    q = torch.full((rows, heads * dim), float("nan"), dtype=DT[act], device="cuda")
    rotary = None
    if rot is not None:
        pos = None if text else torch.randint(0, table_rows, (len(rot[0]), rows), generator=g, device="cuda").to(torch.int32)
        rotary = m.Rotary(m.Rotary.frequencies(table_rows, sum(rot[0])), rot[0], pos, rot[1])
    s = torch.tensor([0] + list(np.cumsum(fresh)), dtype=torch.int32, device="cuda") if starts else None
    n = m.QKNorm(torch.randn(dim, generator=g, device="cuda"), torch.randn(dim, generator=g, device="cuda"), EPS) if norm else None
    return x, q, n, s, rotary


def call(c, heads, x, q, n, s, rotary, **kw):
    if n is None:
        m.mosaic_cache_append(c, x, heads, q, starts=s, rotary=rotary, **kw)
    else:
        m.mosaic_cache_append_norm(c, x, heads, q, n, starts=s, rotary=rotary, **kw)


def step_by_step(x, heads, kv, dim, n, rotary, seen, fresh, dtype):
    """Queries and keys (rows x heads + kv x dim) with every step rounded to
    ``dtype``, and the values; float64 is the formula."""
    x = f64(x).reshape(-1, heads + 2 * kv, dim)
    y = x[:, : heads + kv].astype(dtype)
    if n is not None:
        square = (x[:, : heads + kv] ** 2).mean(axis=-1, keepdims=True)
        w = np.concatenate([np.broadcast_to(f64(t), (k, dim)) for t, k in ((n.q_weight, heads), (n.k_weight, kv))])
        y = y * (1.0 / np.sqrt(square + n.eps)).astype(dtype) * w.astype(dtype)
    if rotary is None:
        return y, x[:, heads + kv:]
    P = sum(rotary.sections)
    out = y.copy()
    table = rotary.table.cpu().numpy().astype(dtype)
    if rotary.positions is None:
        at = np.concatenate([np.arange(s, s + k) for s, k in zip(seen, fresh)]) if fresh else np.zeros(0, np.int64)
        places = np.broadcast_to(at, (len(rotary.sections), len(at)))
    else:
        places = rotary.positions.cpu().numpy()
    j = 0
    for axis, count in enumerate(rotary.sections):
        for _ in range(count):
            lo, hi = (2 * j, 2 * j + 1) if rotary.interleaved else (j, P + j)
            row = np.clip(places[axis], 0, len(table) - 1)
            cs, sn = table[row, j][:, None], table[row, P + j][:, None]
            out[:, :, lo] = y[:, :, lo] * cs - y[:, :, hi] * sn
            out[:, :, hi] = y[:, :, hi] * cs + y[:, :, lo] * sn
            j += 1
    return out, x[:, heads + kv:]


def sizes(x, heads, kv, dim, n, rotary):
    """|y c| + |z s| at most of every element: 1 for cosines and sines."""
    y = np.abs(step_by_step(x, heads, kv, dim, n, None, None, None, np.float64)[0])
    out = y.copy()
    if rotary is not None:
        P = sum(rotary.sections)
        for j in range(P):
            lo, hi = (2 * j, 2 * j + 1) if rotary.interleaved else (j, P + j)
            out[:, :, lo] = out[:, :, hi] = y[:, :, lo] + y[:, :, hi]
    return out


def near(got, want, size, store):
    tol = 8 * U * size + UNIT[store] * np.abs(want) + TINY[store]
    assert got.shape == want.shape and (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


def check(c, old, heads, dim, act, fresh, x, q, n, rotary, util, cache=None):
    """Everything that the call may have written, and that it wrote nothing else.
    Returns the state that it should give."""
    KV, page = c.k.shape[1], c.k.shape[2]
    held, seen = old.state.tolist()
    exact, values = step_by_step(x, heads, KV, dim, n, rotary, seen, fresh, np.float64)
    stepped, _ = step_by_step(x, heads, KV, dim, n, rotary, seen, fresh, np.float32)
    size = sizes(x, heads, KV, dim, n, rotary)
    near(f64(q).reshape(-1, heads, dim), exact[:, :heads], size[:, :heads], act)
    if act == "f32":
        assert np.array_equal(q.cpu().numpy().reshape(-1, heads, dim), stepped[:, :heads])
    want = util.clone(old)
    t = 0
    for b, k in enumerate(fresh):
        fit = max(0, min(k, c.slots - held[b]))
        i = held[b] + torch.arange(fit, device="cuda")
        at, off = c.block_table[b].long()[i // page], i % page
        for name, rows in (("k", stepped[t: t + fit, heads:]), ("v", values[t: t + fit])):
            if cache is None:
                rows = oc.pack_e2m1(*oc.to_e2m1(rows))
                used = dim // 2 + dim // 8
                getattr(want, name)[at, :, off] = torch.cat([torch.from_numpy(rows[..., :used]).cuda(),
                                                             getattr(old, name)[at, :, off][..., used:]], dim=-1)
            else:
                got = getattr(c, name)[at, :, off]
                if name == "k":
                    near(f64(got), exact[t: t + fit, heads:], size[t: t + fit, heads:], cache)
                else:
                    near(f64(got), rows, np.zeros_like(rows), cache)
                getattr(want, name)[at, :, off] = got
        if c.weights is not None:
            want.weights[at, :, off] = 0.0
            want.order[at, :, off] = (seen[b] + i - held[b]).to(torch.int32)[:, None].expand(-1, KV)
        want.state[0, b], want.state[1, b] = held[b] + fit, seen[b] + k
        t += k
    for name in ("k", "v", "weights", "order"):
        if getattr(c, name) is not None:
            assert same_bits(getattr(c, name), getattr(want, name)), name
    return want.state


@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("dim,rot", CASES, ids=lambda v: str(v).replace(" ", ""))
def test_pieces_of_prompts(act, cache, dim, rot):
    """Ragged numbers of new tokens behind held ones, none for a sequence."""
    fresh = (3, 0, 37, 1)
    c = cu.make_cache((0, 5, 30, 16), 2, dim, 16, cache, 7, room=40, evicts=True, seen=(0, 9, 31, 300),
                      layout="tokens" if dim == 80 else "heads")
    old = cu.clone(c)
    args = inputs(c, dim, 6, act, fresh, rot, 8)
    call(c, 6, *args)
    x, q, n, _, rotary = args
    assert torch.equal(c.state, check(c, old, 6, dim, act, fresh, x, q, n, rotary, cu, cache))


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("norm", (False, True))
@pytest.mark.parametrize("dim,rot", CASES, ids=lambda v: str(v).replace(" ", ""))
def test_pieces_of_prompts_in_4_bits(act, norm, dim, rot):
    fresh = (3, 0, 37, 1)
    c = eu.make_cache((0, 5, 30, 16), 2, dim, 16, 7, room=40, evicts=True, seen=(0, 9, 31, 300),
                      layout="tokens" if dim == 80 else "heads", gap=16 if dim == 64 else 0)
    old = eu.clone(c)
    args = inputs(c, dim, 6, act, fresh, rot, 8, norm=norm)
    call(c, 6, *args)
    x, q, n, _, rotary = args
    assert torch.equal(c.state, check(c, old, 6, dim, act, fresh, x, q, n, rotary, eu))


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv", ((1, 1), (64, 8), (5, 5), (71, 1)))
@pytest.mark.parametrize("four", (False, True))
def test_one_token_each(act, heads, kv, four):
    """A decode step without starts; positions from the state; state elsewhere or in place."""
    util, dim = (eu, 128) if four else (cu, 128)
    lengths = (0, 5, 15, 16, 200)
    c = eu.make_cache(lengths, kv, dim, 16, 17, room=1) if four else cu.make_cache(lengths, kv, dim, 16, act, 17, room=1)
    for own in (False, True):
        old = util.clone(c)
        state = None if own else torch.full_like(c.state, -1)
        args = inputs(c, dim, heads, act, (1,) * 5, ((64,), False), 18, starts=False, text=True)
        call(c, heads, *args, new_state=state)
        x, q, n, _, rotary = args
        want = check(c, old, heads, dim, act, (1,) * 5, x, q, n, rotary, util, None if four else act)
        assert torch.equal(c.state if own else state, want)
        if not own:
            assert torch.equal(c.state, old.state)
            c = old


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("rows,batch", ((257, 1), (300, 7), (4096, 4)))
def test_long_prompts(act, rows, batch):
    """More tokens than one per compute unit, and more than the caches hold."""
    fresh = [rows // batch] * batch
    fresh[0] += rows - sum(fresh)
    c = eu.make_cache((3,) * batch, 8, 128, 64, 27, room=max(fresh))
    old = eu.clone(c)
    args = inputs(c, 128, 16 if rows < 4096 else 32, act, fresh, ((64,), False), 28, text=True, table_rows=5000)
    heads = 16 if rows < 4096 else 32
    call(c, heads, *args)
    x, q, n, _, rotary = args
    assert torch.equal(c.state, check(c, old, heads, 128, act, fresh, x, q, n, rotary, eu))


def test_no_room_left():
    """Tokens beyond the last slot are not kept, their queries still written."""
    for starts in (False, True):
        fresh = (9, 2, 1) if starts else (1, 1, 1)
        c = eu.make_cache((10, 16, 16), 2, 64, 16, 27, evicts=True)
        old = eu.clone(c)
        args = inputs(c, 64, 4, "f32", fresh, ((32,), False), 28, starts=starts, text=True)
        call(c, 4, *args)
        x, q, n, _, rotary = args
        assert torch.equal(c.state, check(c, old, 4, 64, "f32", fresh, x, q, n, rotary, eu))


def test_pages_that_are_not_there():
    """Nothing of their tokens is written, the others' are."""
    c = eu.make_cache((10, 30), 2, 64, 16, 37, room=20, evicts=True)
    full = eu.clone(c)
    args = inputs(c, 64, 4, "f32", (3, 5), None, 38)
    call(full, 4, *args)
    c.block_table[0, 0], c.block_table[1, 2] = -1, c.k.shape[0]
    want = eu.clone(c)
    call(c, 4, *args)
    p = int(c.block_table[1, 1])                      # slots 30 and 31 of the second sequence
    for name in ("k", "v", "weights", "order"):
        getattr(want, name)[p, :, 14:16] = getattr(full, name)[p, :, 14:16]
        assert same_bits(getattr(c, name), getattr(want, name)), name
    assert c.state.tolist() == [[13, 35], [13, 35]]


def special(act):
    """Rows of 8: borders between codes, magnitudes over 6, tiny and huge ones,
    zeros of both signs, infinities and NaN."""
    rows = [[0.0] * 8, [-0.0] * 8, [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], [-0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0],
            [7.0] + [0.25] * 7, [7.0 * (1 + UNIT[act] * 2)] + [0.25, 0.5, 0.75] * 2 + [5.0], [3.5, 1.75, 0.875] + [0.1] * 5,
            [3.5 * (1 + UNIT[act] * 2)] + [0.6] * 7, [float("inf")] + [1.0] * 7, [1.0] * 7 + [float("-inf")],
            [1.0, float("nan")] + [2.0] * 6, [float("nan")] * 8]
    if act != "f16":
        most = float(torch.finfo(DT[act]).max)
        rows += [[most, -most] + [1.0] * 6, [2.0 ** 127 * 1.75] + [2.0 ** 125] * 7, [2.0 ** -126] * 8, [2.0 ** -127, -(2.0 ** -126)] * 4,
                 [2.0 ** -130] * 8, [7.0 * 2.0 ** -126] + [2.0 ** -128] * 7, [2.0 ** 100] + [2.0 ** -100] * 7]
    else:
        rows += [[65504.0, -65504.0] + [1.0] * 6, [2.0 ** -24] * 8, [2.0 ** -14] * 8]
    return torch.tensor(rows, dtype=torch.float64).to(DT[act])


@pytest.mark.parametrize("act", eu.ACTS)
def test_special_numbers_in_4_bits(act):
    """Without norms and positions a row is what it says: exactly the oracle's bytes."""
    x8 = special(act)
    n = len(x8)
    c = eu.make_cache((0,), 1, 8, 16, 47, room=n)
    x = torch.zeros((n, 3 * 8), dtype=DT[act], device="cuda")
    x[:, 8: 16], x[:, 16:] = x8.cuda(), x8.flip(1).cuda()
    q = torch.empty((n, 8), dtype=DT[act], device="cuda")
    m.mosaic_cache_append(c, x, 1, q, starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    for name, want in (("k", x8), ("v", x8.flip(1))):
        got = eu.rows_of(c, name, 0, 0, n)[0]
        codes, scales = oc.to_e2m1(want.double().numpy())
        wrote = np.stack([got[:, :4] % 16, got[:, :4] // 16], axis=-1).reshape(n, 8)
        # the sign of a zero says nothing
        assert np.array_equal(np.where(wrote % 8 == 0, 0, wrote), np.where(codes % 8 == 0, 0, codes))
        assert np.array_equal(got[:, 4:5], scales)


@pytest.mark.parametrize("act,cache", (("f32", "f32"), ("bf16", "bf16"), ("f32", "4")))
def test_heads_without_a_norm(act, cache):
    """Heads of zeros, of an infinity and of NaN act as in the formulas; the
    others do not notice."""
    util, c = (eu, eu.make_cache((2,), 2, 64, 16, 57, room=4)) if cache == "4" else \
        (cu, cu.make_cache((2,), 2, 64, 16, cache, 57, room=4))
    x, q, n, s, rotary = inputs(c, 64, 4, act, (4,), None, 58)
    x[1, :64], x[2, 64: 128] = 0.0, 0.0
    x[2, 70], x[3, 130] = float("inf"), float("nan")
    x[1, 256 + 3] = float("-inf")                     # a key
    call(c, 4, x, q, n, s, rotary)
    with np.errstate(invalid="ignore"):
        want, _ = step_by_step(x, 4, 2, 64, n, None, (2,), (4,), np.float64)
    got = f64(q).reshape(4, 4, 64)
    assert not got[1, 0].any()
    assert np.array_equal(np.isnan(got), np.isnan(want[:, :4])) and np.isnan(got[2, 1]).sum() == 1
    ok = ~np.isnan(want[:, :4])
    assert (np.abs(got - want[:, :4])[ok] <= (4 * U + UNIT[act]) * np.abs(want[:, :4])[ok]).all()
    k = util.get(c, "k", 0, 6)[:, 2:]
    bad = np.isnan(k)
    assert bad[0, 1].sum() == (8 if cache == "4" else 1) and bad.sum() == bad[0, 1].sum()


def test_strided_rows():
    c = eu.make_cache((3, 20), 2, 64, 16, 67, room=8, gap=32)
    want = eu.clone(c)
    x, q, n, s, rotary = inputs(c, 64, 4, "f16", (2, 5), ((20, 12), False), 68)
    call(want, 4, x, q, n, s, rotary)
    wide_x = torch.zeros((7, 640), dtype=torch.float16, device="cuda")
    wide_q = torch.zeros((9, 320), dtype=torch.float16, device="cuda")
    wide_x[:, 64: 576] = x
    call(c, 4, wide_x[:, 64: 576], wide_q[:7, 8: 264], n, s, rotary)
    assert torch.equal(wide_q[:7, 8: 264], q) and not wide_q[:, :8].any() and not wide_q[:, 264:].any()
    assert not wide_q[7:].any()
    assert torch.equal(c.k, want.k) and torch.equal(c.v, want.v) and torch.equal(c.state, want.state)


def test_nothing_new():
    """No rows at all: only the state is handed on; no sequence: nothing is."""
    c = eu.make_cache((3, 4), 2, 64, 16, 69)
    old, state = eu.clone(c), torch.full_like(c.state, -1)
    w = torch.ones(64, device="cuda")
    x, q = torch.empty((0, 8 * 64), device="cuda"), torch.empty((0, 256), device="cuda")
    m.mosaic_cache_append_norm(c, x, 4, q, m.QKNorm(w, w), starts=torch.zeros(3, dtype=torch.int32, device="cuda"),
                               new_state=state)
    assert torch.equal(state, old.state) and torch.equal(c.k, old.k) and torch.equal(c.v, old.v)
    none = eu.make_cache((), 2, 64, 16, 70)
    m.mosaic_cache_append_norm(none, x, 4, q, m.QKNorm(w, w))
    m.mosaic_cache_attend(none, q, 4, torch.empty_like(q))
    m.mosaic_cache_read(none, torch.empty((0, 128), device="cuda"), torch.empty((0, 128), device="cuda"))


def test_state_elsewhere_with_starts():
    """Ragged tokens with the new state in another tensor, several tokens to a workgroup."""
    fresh = (700, 0, 900, 3)
    c = eu.make_cache((5, 9, 0, 30), 2, 64, 64, 71, room=900)
    old, state = eu.clone(c), torch.full_like(c.state, -1)
    args = inputs(c, 64, 4, "bf16", fresh, ((32,), False), 72, text=True, table_rows=1000)
    call(c, 4, *args, new_state=state)
    x, q, n, _, rotary = args
    assert torch.equal(state, check(c, old, 4, 64, "bf16", fresh, x, q, n, rotary, eu)) and torch.equal(c.state, old.state)


def test_many_sequences_of_one_token():
    """More sequences than a workgroup per compute unit, no starts, state in place."""
    batch = 1300
    lengths = [int(i) for i in np.random.default_rng(5).integers(0, 40, batch)]
    c = eu.make_cache(lengths, 1, 16, 16, 73, room=1)
    old = eu.clone(c)
    args = inputs(c, 16, 2, "f16", (1,) * batch, ((8,), False), 74, starts=False, text=True)
    call(c, 2, *args)
    x, q, n, _, rotary = args
    assert torch.equal(c.state, check(c, old, 2, 16, "f16", (1,) * batch, x, q, n, rotary, eu))


@pytest.mark.parametrize("four", (False, True))
def test_graph_of_a_step(four):
    """Captured with the state in place, on a stream of its own: every replay is
    the next token."""
    util = eu if four else cu
    c = eu.make_cache((14, 3), 2, 64, 16, 77, room=10, evicts=True) if four else \
        cu.make_cache((14, 3), 2, 64, 16, "bf16", 77, room=10, evicts=True)
    want = util.clone(c)
    x, q, n, _, rotary = inputs(c, 64, 4, "f32", (1, 1), ((32,), False), 78, starts=False, text=True)
    q2 = torch.empty_like(q)
    call(c, 4, x, q, n, None, rotary)
    call(want, 4, x, q2, n, None, rotary)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c, 4, x, q, n, None, rotary)
    for step in range(4):
        x.copy_(torch.randn(x.shape, generator=seeded(80 + step), device="cuda"))
        graph.replay()
        call(want, 4, x, q2, n, None, rotary)
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and torch.equal(c.state, want.state)
        for name in ("k", "v", "weights", "order"):
            assert same_bits(getattr(c, name), getattr(want, name)), name


def test_refusals():
    c = eu.make_cache((3, 4), 2, 64, 16, 87, room=4)
    x, q = torch.zeros((2, 512), device="cuda"), torch.zeros((2, 256), device="cuda")
    w = torch.ones(64, device="cuda")
    def go(x=x, heads=4, q=q, norm=m.QKNorm(w, w), c=c, **kw):
        m.mosaic_cache_append_norm(c, x, heads, q, norm, **kw)
    go()
    for bad in (dict(heads=3), dict(norm=m.QKNorm(w, w, -1.0)), dict(norm=m.QKNorm(w, w, float("nan"))),
                dict(norm=m.QKNorm(w, w, float("inf")))):
        with pytest.raises(m.MosaicError) as e:
            go(**bad)
        assert e.value.status == m.STATUS_INVALID_ARG
    short = m.KVCache(c.k[..., :32], c.v[..., :32], c.block_table, c.state, head_dim=64)
    unsaid = m.KVCache(c.k, c.v, c.block_table, c.state)
    for bad in (dict(norm=m.QKNorm(w[:56], w)), dict(norm=m.QKNorm(w, w.double())), dict(norm=m.QKNorm(w.cpu(), w)),
                dict(norm=m.QKNorm(w, torch.ones(128, device="cuda")[::2])), dict(x=x[:, :448]), dict(q=q.bfloat16()),
                dict(x=x.double(), q=q.double()), dict(c=short), dict(c=unsaid)):
        with pytest.raises(ValueError):
            go(**bad)
