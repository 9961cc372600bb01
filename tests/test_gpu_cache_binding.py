"""The two ways from the Python functions of the cached decoding into the C ABI,
native marshalling and ctypes, give the same bits."""
import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests.cache_util import DT, TYPES, clone, make_cache, same_bits, seeded

pytestmark = pytest.mark.gpu


class _Declines:
    """Stands in for the native marshalling; counts the arguments it was handed."""

    def __init__(self):
        self.handed = []

    def cache_append(self, *args):
        self.handed.append(len(args))

    cache_attend = cache_evict = cache_append


def _step(c, act, starts, out_of_place):
    g = seeded(3)
    x = torch.randn((5, 8 * 64), generator=g, device="cuda").to(DT[act])
    q = torch.empty((5, 256), dtype=DT[act], device="cuda")
    rotary = m.Rotary(m.Rotary.frequencies(64, 32), [8, 12, 12],
                      torch.randint(0, 64, (3, 5), generator=g, device="cuda", dtype=torch.int32), True)
    m.mosaic_cache_append(c, x, 4, q, starts=starts, rotary=rotary)
    out = torch.empty((c.batch, 256), dtype=DT[act], device="cuda")
    m.mosaic_cache_attend(c, q[: c.batch], 4, out, max_len=60, scale=0.2, accumulate=True)
    kept = torch.empty((c.batch, 2, 30), dtype=torch.int32, device="cuda")
    new = dict(new_state=torch.zeros_like(c.state), new_weights=torch.zeros_like(c.weights),
               new_order=torch.zeros_like(c.order)) if out_of_place else {}
    m.mosaic_cache_evict(c, 30, 4, max_len=60, kept=kept, **new)
    return [q, out, kept, c.k, c.v, c.weights, c.order, c.state, *new.values()]


@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("apart", (False, True))
def test_both_ways_agree(monkeypatch, act, cache, apart):
    c = make_cache((3, 40, 17), 2, 64, 16, cache, 5, room=4, evicts=True)
    starts = torch.tensor([0, 1, 1, 5], dtype=torch.int32, device="cuda")
    other = clone(c)
    want = _step(c, act, starts, apart)
    declines = _Declines()
    monkeypatch.setattr(m, "_b", declines)
    got = _step(other, act, starts, apart)
    assert declines.handed == [7, 7, 8]
    assert all(same_bits(a, b) for a, b in zip(got, want))


def test_native_takes_well_formed_calls():
    """No status is None: the ctypes code is not what runs by default."""
    b = m._native()
    c = make_cache((3, 40), 2, 64, 16, "bf16", 6, room=4, evicts=True)
    x, q = torch.zeros((2, 512), device="cuda"), torch.zeros((2, 256), device="cuda")
    assert b.cache_append(c, x, 4, q, None, m.Rotary(m.Rotary.frequencies(64, 32), (32,)), None) == 0
    assert b.cache_attend(c, q, 4, torch.empty_like(q), None, None, True) == 0
    assert b.cache_evict(c, 20, 2, 50, None, None, None, None) == 0
    assert b.cache_attend(c, q.cpu(), 4, q, None, None, True) is None
    assert b.cache_attend(c, q, 4, q[:1], None, None, True) is None
    assert b.cache_attend(object(), q, 4, q, None, None, True) is None
    assert b.cache_append(c, x, 4.0, q, None, None, None) is None
    assert b.cache_evict(c, 0, 0, None, None, None, None, None) is None
    torch.cuda.synchronize()
