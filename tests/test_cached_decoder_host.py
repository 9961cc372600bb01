"""What CachedDecoder keeps count of and refuses, without a GPU: the operators
are replaced by ones that advance the caches' state."""
import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from paper_2607_29221_amd.cached_decoder import CachedDecoder

CFG = dict(hidden=8, heads=2, kv_heads=1, head_dim=8, ffn=4, layers=2, batch=2, seq=5)
WIDTH = {"qkv": 32, "o": 8, "gate_up": 8, "down": 8}


@pytest.fixture(autouse=True)
def operators(monkeypatch):
    def append(cache, qkv, heads, q_out, starts=None, rotary=None, new_state=None):
        q_out.zero_()
        cache.state += qkv.shape[0] // cache.batch

    def attend(cache, q, heads, out, max_len=None, scale=None, accumulate=False):
        assert max_len == int(cache.state[0].max())
        out.zero_()

    def evict(cache, budget, recent, max_len=None, **kw):
        assert max_len == int(cache.state[0].max())
        cache.state[0].clamp_(max=budget)
    for name, f in (("append", append), ("attend", attend), ("evict", evict)):
        monkeypatch.setattr(m, "mosaic_cache_" + name, f)


def linear(layer, name, x):
    return torch.zeros(x.shape[0], WIDTH[name])


def decoder(max_len=64, lin=linear, **kw):
    return CachedDecoder(lin, 2, CFG, max_len, page_size=16, device="cpu", **kw)


def rows(n):
    return torch.zeros(2 * n, 8)


@pytest.mark.parametrize("budget", (None, 4))
def test_numbers_beyond_the_rotary_table(budget):
    """With a budget the tokens held stay few while their numbers go on."""
    table = m.Rotary.frequencies(10, 4, device="cpu")
    d = decoder(table=table, sections=[4], budget=budget)
    with pytest.raises(ValueError, match="rotary table"):
        d.prompt(rows(11))
    d.prompt(rows(7))
    for _ in range(3):
        d.step(rows(1))
    assert d.seen == 10 and d.held == (10 if budget is None else 4)
    with pytest.raises(ValueError, match="rotary table"):
        d.step(rows(1))
    assert d.seen == 10
    d.step(rows(1), positions=torch.tensor([[3, 9]], dtype=torch.int32))      # places of the caller's
    with pytest.raises(ValueError, match="rotary table"):
        d.step(rows(1))
    free = decoder(budget=budget)                                              # nothing is turned
    free.prompt(rows(30))
    free.step(rows(1))


@pytest.mark.gpu
def test_on_the_device(monkeypatch):
    """The device's count is the decoder's."""
    monkeypatch.undo()
    table = m.Rotary.frequencies(10, 4)
    d = CachedDecoder(lambda layer, name, x: torch.zeros(x.shape[0], WIDTH[name], device="cuda"), 2, CFG, 64,
                      page_size=16, budget=4, table=table, sections=[4])
    d.prompt(rows(7).cuda())
    for _ in range(3):
        d.step(rows(1).cuda())
    assert all(c.state.tolist() == [[4, 4], [10, 10]] for c in d.caches) and d.seen == 10
    with pytest.raises(ValueError, match="rotary table"):
        d.step(rows(1).cuda())


@pytest.mark.parametrize("budget", (0, -1))
def test_a_budget_of_nothing(budget):
    """Refused at once, not in the first layer that evicts."""
    with pytest.raises(ValueError, match="budget"):
        decoder(budget=budget)


@pytest.mark.parametrize("max_len", (32, 30, 48))
def test_as_many_slots_as_the_budget(max_len):
    """A decode at its budget goes on without end; max_len 30 makes 32 slots."""
    d = decoder(max_len, budget=32)
    d.prompt(rows(31))
    for _ in range(10):
        d.step(rows(1))
    assert d.held == 32 and d.seen == 41


def test_a_budget_beyond_the_slots():
    d = decoder(32, budget=33)
    d.prompt(rows(31))
    d.step(rows(1))
    with pytest.raises(ValueError, match="no slot"):
        d.step(rows(1))


class _Fails:
    """Linear layers of which one raises once."""

    def __init__(self, layer, name):
        self.at = (layer, name)

    def __call__(self, layer, name, x):
        if (layer, name) == self.at:
            self.at = None
            raise ConnectionError("no answer")
        return linear(layer, name, x)


WHERE = [(layer, name) for layer in range(2) for name in WIDTH]


def states(d):
    return [c.state.tolist() for c in d.caches]


@pytest.mark.parametrize("layer,name", WHERE)
@pytest.mark.parametrize("budget", (None, 4, 40))
def test_a_prompt_that_fails_can_be_made_again(layer, name, budget):
    d = decoder(lin=_Fails(layer, name), budget=budget)
    with pytest.raises(ConnectionError):
        d.prompt(rows(7))
    assert d.held == d.seen == 0 and states(d) == [[[0, 0], [0, 0]]] * 2
    d.prompt(rows(6))
    n = 6 if budget != 4 else 4
    assert d.held == n and d.seen == 6 and states(d) == [[[n, n], [6, 6]]] * 2


@pytest.mark.parametrize("layer,name", WHERE)
@pytest.mark.parametrize("budget", (None, 4, 40))
def test_a_step_that_fails(layer, name, budget):
    d = decoder(budget=budget)
    d.prompt(rows(7))
    before = states(d)
    d.linear = _Fails(layer, name)
    with pytest.raises(ConnectionError):
        d.step(rows(1))
    if budget is not None and (layer, name) != (0, "qkv"):
        for call in (d.step, d.prompt):
            with pytest.raises(RuntimeError, match="cannot be used"):
                call(rows(1))
        return
    assert d.seen == 7 and states(d) == before
    d.step(rows(1))
    n = 8 if budget != 4 else 4
    assert d.held == n and d.seen == 8 and states(d) == [[[n, n], [8, 8]]] * 2


@pytest.mark.gpu
def test_a_failed_step_on_the_device(monkeypatch):
    """The same hidden states with a failure in between as without."""
    monkeypatch.undo()
    g = torch.Generator(device="cuda").manual_seed(5)
    w = {n: torch.randn((o, 4 if n == "down" else 8), generator=g, device="cuda") for n, o in
         (("qkv", 32), ("o", 8), ("gate_up", 8), ("down", 8))}
    w["o"] = torch.randn((8, 16), generator=g, device="cuda")
    x = torch.randn((2 * 9, 8), generator=g, device="cuda")
    table = m.Rotary.frequencies(10, 4)

    def lin(layer, name, a):
        return a @ w[name].t()

    def run(fail):
        d = CachedDecoder(lin, 2, CFG, 64, page_size=16, table=table, sections=[4])
        outs = []
        for part in (x[:14], x[14:16], x[16:]):
            call = d.prompt if part.shape[0] > 2 else d.step
            if fail:
                failing = _Fails(1, "gate_up")
                d.linear = lambda l, n, a: failing(l, n, a) if (l, n) == failing.at else lin(l, n, a)
                with pytest.raises(ConnectionError):
                    call(part + 1.0)
                d.linear = lin
            outs.append(call(part))
        return torch.cat(outs)
    assert torch.equal(run(False), run(True))
