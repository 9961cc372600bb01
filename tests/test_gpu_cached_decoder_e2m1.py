"""Decoding with caches in 4 bits and with norms of queries and keys: against
the whole forward in float64 on the keys and values that 4 bits hold for it."""
import math

import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import decoder as dec
from paper_2607_29221_amd import mosaic as m
from paper_2607_29221_amd.cached_decoder import CachedDecoder
from tests.test_gpu_cached_decoder import CFG, plain, run, stack

pytestmark = pytest.mark.gpu


def norms():
    g = torch.Generator(device="cuda").manual_seed(7)
    return [m.QKNorm(*(1.0 + 0.3 * torch.randn(CFG["head_dim"], generator=g, device="cuda") for _ in range(2)), 1e-5)
            for _ in range(CFG["layers"])]


def reference(weights, x, table, qk, held=None):
    """All tokens in float64, layer by layer; held(x): what the cache makes of keys and values."""
    B, S, H = x.shape
    heads, kv, D, F = CFG["heads"], CFG["kv_heads"], CFG["head_dim"], CFG["ffn"]
    P = D // 2
    cos, sin = table[:S, :P].double()[:, None, :], table[:S, P:].double()[:, None, :]

    def rms(a, eps=1e-5):
        return a / torch.sqrt((a * a).mean(-1, keepdim=True) + eps)

    def turn(a):
        u, v = a[..., :P], a[..., P:]
        return torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    h = x.double()
    for l, layer in enumerate(weights):
        W = {n: w.double() for n, w in layer.items()}
        qkv = (rms(h) @ W["qkv"].t()).reshape(B, S, heads + 2 * kv, D)
        q, k, v = qkv[:, :, :heads], qkv[:, :, heads: heads + kv], qkv[:, :, heads + kv:]
        if qk is not None:
            eps = float(torch.tensor(qk[l].eps, dtype=torch.float32))
            q, k = rms(q, eps) * qk[l].q_weight.double(), rms(k, eps) * qk[l].k_weight.double()
        q, k = turn(q), turn(k)
        if held is not None:
            k, v = held(k), held(v)
        a = torch.empty_like(q)
        mask = torch.ones((S, S), dtype=torch.bool, device=x.device).triu(1)
        for b in range(B):
            for g in range(heads):
                s = (q[b, :, g] @ k[b, :, g // (heads // kv)].t()) / math.sqrt(D)
                a[b, :, g] = torch.softmax(s.masked_fill(mask, float("-inf")), -1) @ v[b, :, g // (heads // kv)]
        h = h + a.reshape(B, S, heads * D) @ W["o"].t()
        gu = rms(h) @ W["gate_up"].t()
        h = h + (torch.nn.functional.silu(gu[..., :F]) * gu[..., F:]) @ W["down"].t()
    return h


def four_bits(t):
    return torch.from_numpy(oc.unpack_e2m1(oc.pack_e2m1(*oc.to_e2m1(t.cpu().numpy())), t.shape[-1])).to(t.device)


@pytest.mark.parametrize("prompt", (1, 17, 39))
@pytest.mark.parametrize("normed", (False, True))
def test_float32_cache_with_norms(prompt, normed):
    """The same bound as without norms: two layers of products of at most 512
    terms, each off by its rounding (512 u = 3e-5 at worst)."""
    weights, x = stack()
    table, qk = m.Rotary.frequencies(64, 32), norms() if normed else None
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], page_size=16, table=table, sections=[32], norms=qk)
    e = dec.error_metrics(run(d, x, prompt), reference(weights, x, table, qk).float())
    assert e["rel_l2"] < 3e-5, e


@pytest.mark.parametrize("prompt", (1, 17, 39))
@pytest.mark.parametrize("normed", (False, True))
def test_cache_in_4_bits(prompt, normed):
    """Float32 keys differ from float64 ones by 1e-6 of their size at most, so one
    code in 1e5 or so falls on the other side of its border: of the 2 x 2 x 40 x 2 x
    2 x 64 = 40960 elements held a few, each a step of at most a third of the
    element. One such key or value moves a token's output by a 1 / sqrt(64 tokens)
    part of the quantisation's own effect; 1e-3 leaves room for a dozen."""
    weights, x = stack()
    table, qk = m.Rotary.frequencies(64, 32), norms() if normed else None
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], dtype=torch.uint8, page_size=16, table=table,
                      sections=[32], norms=qk)
    got = run(d, x, prompt)
    e = dec.error_metrics(got, reference(weights, x, table, qk, four_bits).float())
    assert e["rel_l2"] < 1e-3, e
    # and the 4 bits are what moves it from the float32 decode: by 0.2 of an element at most
    far = dec.error_metrics(got, reference(weights, x, table, qk).float())
    assert 1e-3 < far["rel_l2"] < 0.2, far


def test_budget_in_4_bits():
    """A prompt cut to a budget, then steps that each evict a token: the caches
    hold the budget, and a budget that is never reached changes nothing."""
    weights, x = stack()
    table = m.Rotary.frequencies(64, 32)
    outs = []
    for budget in (None, 64, 16):
        d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"] + 24, dtype=torch.uint8, page_size=16, table=table,
                          sections=[32], norms=norms(), budget=budget, recent=0 if budget is None else 4)
        outs.append(run(d, x, 20))
        assert d.held == (16 if budget == 16 else CFG["seq"])
        assert all(c.state[0].tolist() == [d.held] * 2 and c.state[1].tolist() == [CFG["seq"]] * 2 for c in d.caches)
    assert torch.isfinite(outs[2]).all()
    assert torch.equal(outs[0][:, :20], outs[1][:, :20])
    e = dec.error_metrics(outs[1], outs[0])          # the weights' sums alone differ in the making
    assert e["rel_l2"] < 1e-5, e
    assert torch.equal(outs[2][:, :20], outs[0][:, :20]) and not torch.equal(outs[2], outs[0])


def test_norms_of_other_layers_are_refused():
    with pytest.raises(ValueError, match="norms"):
        CachedDecoder(lambda *a: None, 3, CFG, 16, norms=norms())
