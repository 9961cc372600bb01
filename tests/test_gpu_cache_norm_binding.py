"""Norms, caches in 4 bits and cached rows through native marshalling and through
ctypes: the same bits; both refuse a cache that is not on the current device."""
import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests import e2m1_util as eu
from tests.cache_util import DT, same_bits, seeded

pytestmark = pytest.mark.gpu


class _Declines:
    """Stands in for the native marshalling; counts the arguments it was handed."""

    def __init__(self):
        self.handed = []

    def cache_append(self, *args):
        self.handed.append(len(args))

    cache_append_norm = cache_read = cache_attend = cache_evict = cache_append


def _step(c, act):
    g = seeded(3)
    x = torch.randn((5, 8 * 64), generator=g, device="cuda").to(DT[act])
    q, q2 = (torch.empty((5, 256), dtype=DT[act], device="cuda") for _ in range(2))
    starts = torch.tensor([0, 1, 1, 5], dtype=torch.int32, device="cuda")
    first = c.state[0].clone()
    rotary = m.Rotary(m.Rotary.frequencies(64, 32), [8, 12, 12],
                      torch.randint(0, 64, (3, 5), generator=g, device="cuda", dtype=torch.int32), True)
    w = torch.rand(64, generator=g, device="cuda")
    m.mosaic_cache_append_norm(c, x, 4, q, m.QKNorm(w, w + 1.0, 0.01), starts=starts, rotary=rotary)
    m.mosaic_cache_append(c, x, 4, q2, starts=starts)
    k, v = (torch.empty((10, 128), dtype=DT[act], device="cuda") for _ in range(2))
    m.mosaic_cache_read(c, k, v, starts=2 * starts, first=first)
    out = torch.empty((3, 256), dtype=DT[act], device="cuda")
    m.mosaic_cache_attend(c, q[:3], 4, out, max_len=60, scale=0.2, accumulate=True)
    kept = torch.empty((3, 2, 30), dtype=torch.int32, device="cuda")
    m.mosaic_cache_evict(c, 30, 4, max_len=60, kept=kept)
    return [q, q2, k, v, out, kept, c.k, c.v, c.weights, c.order, c.state]


@pytest.mark.parametrize("act", eu.ACTS)
def test_both_ways_agree(monkeypatch, act):
    c = eu.make_cache((3, 40, 17), 2, 64, 16, 5, room=9, evicts=True)
    other = eu.clone(c)
    want = _step(c, act)
    declines = _Declines()
    monkeypatch.setattr(m, "_b", declines)
    got = _step(other, act)
    assert declines.handed == [8, 7, 5, 7, 8]
    for a, b in zip(got, want):
        assert same_bits(a, b)


def test_a_whole_number_for_eps():
    """Not a float: declined by the native marshalling, taken by the other."""
    c = eu.make_cache((3,), 2, 64, 16, 6, room=2)
    x, q, w = torch.ones((1, 512), device="cuda"), torch.empty((1, 256), device="cuda"), torch.ones(64, device="cuda")
    m.mosaic_cache_append_norm(c, x, 4, q, m.QKNorm(w, w, 0))
    assert (q == 1).all()


def test_another_device(monkeypatch):
    """As if the current device were another one; both ways refuse."""
    c = eu.make_cache((3, 4), 2, 64, 16, 7, room=2)
    x, q, w = torch.ones((2, 512), device="cuda"), torch.empty((2, 256), device="cuda"), torch.ones(64, device="cuda")
    rows = torch.empty((2, 128), device="cuda")
    calls = (lambda: m.mosaic_cache_append(c, x, 4, q), lambda: m.mosaic_cache_append_norm(c, x, 4, q, m.QKNorm(w, w)),
             lambda: m.mosaic_cache_read(c, rows, torch.empty_like(rows)), lambda: m.mosaic_cache_attend(c, q, 4, torch.empty_like(q)))
    monkeypatch.setattr(m, "_b", _Declines())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    state = c.state.clone()
    for call in calls:
        with pytest.raises(ValueError, match="device"):
            call()
    assert torch.equal(c.state, state)
