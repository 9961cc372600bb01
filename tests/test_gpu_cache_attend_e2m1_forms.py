"""Every form of the kernel of the attention over 4 bits (heads side by side, one
and several blocks of heads, whole and padded head dimensions), and shares that are
long enough for a sequence's start to count as steps of its own: shares that begin
in these steps, at a sequence's first one and behind empty sequences, in batches of
fewer and of more sequences than a wave has lanes. Tolerances as in
test_gpu_cache_attend_e2m1.py."""
import numpy as np
import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests import e2m1_util as eu
from tests.cache_util import DT, same_bits, seeded
from tests.test_gpu_cache_attend_e2m1 import check, run

pytestmark = pytest.mark.gpu
STEP, START, LONG = 128, 2, 16


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("group", (1, 4, 5, 8, 9, 16, 17, 32, 33))
@pytest.mark.parametrize("dim", (64, 128, 256, 56, 104, 200))
def test_forms(act, accumulate, group, dim):
    lengths = (130, 0, 33, 1)
    c = eu.make_cache(lengths, 2, dim, 32 if group % 2 else 16, 5, evicts=accumulate)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)] if accumulate else None
    q, out, scale = run(c, 2 * group, act, 6, accumulate=accumulate)
    check(c, q, 2 * group, out, act, scale, before)


def workgroups(kv, group):
    """Of a key/value head and block of query heads: two per unit, for heads of up
    to 128 elements whose LDS leaves room for two."""
    tiles = -(-group // 16)
    tiles = -(-tiles // 2) if tiles > 1 else 1
    each = (512 // 8 // tiles * 8 if tiles > 1 else 512) // kv
    assert 16 * each * kv * tiles >= 15 * 512
    return each


def borders(lengths, shares):
    """Where the shares begin, by the formulas of the header: (sequence, step of it)."""
    steps = [-(-n // STEP) for n in lengths]
    assert sum(steps) // shares >= LONG and len(lengths) > 1          # starts count
    ends = np.cumsum([s + START if s else 0 for s in steps])
    share = -(-int(ends[-1]) // shares)
    found = []
    for at in range(share, int(ends[-1]), share):
        b = int(np.searchsorted(ends, at, side="right"))
        found.append((b, at - (int(ends[b - 1]) if b else 0) - steps[b]))
    return found                                                      # the step counted from the sequence's end


def random_cache(lengths, kv, dim, page, seed, evicts=False):
    """As e2m1_util.make_cache, its rows random codes and scales."""
    c = eu.make_cache([0] * len(lengths), kv, dim, page, seed, room=max(lengths), evicts=evicts)
    c.state.copy_(torch.tensor([lengths] * 2, dtype=torch.int32))
    g = seeded(seed + 1)
    for b, n in enumerate(lengths):
        if n:
            p, o = eu.where(c, b, 0, n)
            for t in (c.k, c.v):
                t[p, :, o, :dim // 2] = torch.randint(0, 256, (n, kv, dim // 2), generator=g, device="cuda", dtype=torch.uint8)
                t[p, :, o, dim // 2: dim // 2 + dim // 8] = torch.randint(123, 128, (n, kv, dim // 8), generator=g, device="cuda", dtype=torch.uint8)
            if evicts:
                c.weights[p, :, o] = torch.rand((n, kv), generator=g, device="cuda")
    return c


def shares_and_check(lengths, kv, group, dim, act, accumulate, page=64):
    c = random_cache(lengths, kv, dim, page, 11, evicts=accumulate)
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)] if accumulate else None
    old = eu.clone(c)
    q, out, scale = run(c, kv * group, act, 12, accumulate=accumulate)
    check(c, q, kv * group, out, act, scale, before)
    if accumulate:
        used = torch.zeros_like(c.weights, dtype=torch.bool)
        for b, n in enumerate(lengths):
            p, o = eu.where(c, b, 0, n)
            used[p, :, o] = True
        assert same_bits(c.weights[~used], old.weights[~used])
    again = torch.full_like(out, float("nan"))
    w = eu.clone(old)
    m.mosaic_cache_attend(w, q, kv * group, again, accumulate=accumulate)
    assert torch.equal(out, again)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("kv,group,dim", ((128, 1, 8), (128, 3, 16), (128, 8, 64), (128, 20, 8)))
def test_shares_that_begin_between_sequences(act, accumulate, kv, group, dim):
    """Four shares of S steps: the second begins at the first of the two steps behind
    sequence 0's, the third at the second one behind sequence 1's, the last at the
    first step of sequence 3."""
    S = LONG + 2
    steps = (S, S - 3, S - 3, S - 2)
    for cut in (0, 5) if dim < 64 else (5,):              # whole last steps, and short ones
        lengths = [STEP * s - cut for s in steps]
        assert workgroups(kv, group) == 4
        assert borders(lengths, 4) == [(0, 0), (1, 1), (3, -(S - 2))]
        shares_and_check(lengths, kv, group, dim, act, accumulate)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("accumulate", (False, True))
def test_empty_sequences_among_long_shares(act, accumulate):
    """First, last, and behind a share that begins in a sequence's counted start."""
    S = LONG + 2
    lengths = [0, STEP * S - 100, 0, 0, STEP * (S - 3), 1 + STEP * (S - 4), 0, STEP * (S - 2) - 127, 0]
    assert borders(lengths, 4) == [(1, 0), (4, 1), (7, -(S - 2))]
    shares_and_check(lengths, 128, 2, 8, act, accumulate, page=16)


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("batch", (64, 65, 130, 200))
def test_long_shares_of_many_sequences(act, accumulate, batch):
    """More sequences than lanes; shares begin in the starts of late ones too."""
    r = np.random.default_rng(batch)
    lengths = [int(n) if r.random() < 0.7 else 0 for n in r.integers(1, 700, batch)]
    lengths[batch // 2], lengths[-2], lengths[-1] = 2000, 1290, 640
    kv = 64
    assert workgroups(kv, 2) == 8
    found = borders(lengths, 8)
    assert len(found) == 7 and any(b >= batch // 2 for b, _ in found)
    shares_and_check(lengths, kv, 2, 8, act, accumulate)


@pytest.mark.parametrize("first", range(4))
def test_every_border(first):
    """A share's begin moved step by step across a sequence's end: from its last step
    over the two behind it to the next one's first and second."""
    S = LONG + 4
    seen = set()
    for s0 in range(S - 4, S + 2):
        lengths = [STEP * s0 - 7 * first, STEP * (2 * S - 4 - s0) - first]
        found = borders(lengths, 2)
        seen.add(found[0][1] if found[0][0] == 0 else ("next", found[0][1] + (2 * S - 4 - s0)))
        shares_and_check(lengths, 256, 1, 8, "f32", bool(first % 2))
    assert {-1, 0, 1, ("next", 0), ("next", 1)} <= seen
