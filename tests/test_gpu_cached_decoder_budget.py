"""A prompt longer than the budget through CachedDecoder: the weight that each
token of the prompt got, what the eviction right after the prompt keeps, and
the steps that follow, for every layer, sequence and head."""
import math

import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import decoder as dec
from paper_2607_29221_amd import mosaic as m
from paper_2607_29221_amd.cached_decoder import CachedDecoder
from tests.test_gpu_cached_decoder import CFG, _no_reduced_precision, plain, reference, stack  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def slots(c, b, n):
    page = c.k.shape[2]
    i = torch.arange(n, device="cuda")
    return c.block_table[b].long()[i // page], i % page


@pytest.mark.parametrize("prompt,budget,recent,sharp", ((30, 16, 5, 1), (33, 32, 0, 1), (40, 7, 7, 1), (30, 16, 5, 4)))
def test_a_prompt_beyond_the_budget(monkeypatch, prompt, budget, recent, sharp):
    """``sharp``: a factor of the q|k|v weights. Flat attention gives a prompt's
    first tokens the most, in every head; sharp attention does not."""
    weights, x = stack()
    for layer in weights:
        layer["qkv"] = layer["qkv"] * sharp
    B, S, H = x.shape
    KV, D, G = CFG["kv_heads"], CFG["head_dim"], CFG["heads"] // CFG["kv_heads"]
    table = m.Rotary.frequencies(64, 32)
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"] + 1, page_size=16, table=table, sections=(32,),
                      budget=budget, recent=recent)
    queries, found = [], []
    append, evict = m.mosaic_cache_append, m.mosaic_cache_evict

    def keep_queries(cache, qkv, heads, q_out, **kw):
        append(cache, qkv, heads, q_out, **kw)
        queries.append(q_out.double().view(B, prompt, KV, G, D))

    def check_weights(cache, *args, **kw):
        """What the prompt's attention added up, against float64."""
        before = []
        for b in range(B):
            page, off = slots(cache, b, prompt)
            k = cache.k[page, :, off].double()
            s = torch.stack([queries[-1][b, :, j].transpose(0, 1) @ k[:, j].t() for j in range(KV)]) / math.sqrt(D)
            s.masked_fill_(torch.ones((prompt, prompt), dtype=torch.bool, device="cuda").triu_(1), -math.inf)
            p = torch.softmax(s, dim=-1)                                   # kv x group x queries x tokens
            size = torch.stack([queries[-1][b, :, j].abs().transpose(0, 1) @ k[:, j].abs().t() for j in range(KV)])
            # a weight's own error as in test_gpu_cache_attend.py, and a float32 sum over group and queries
            rel = (2 * (D + 4) * size.amax() / math.sqrt(D) + prompt + 16 + G * prompt) * U
            got = cache.weights[page, :, off].double().t()
            assert ((got - p.sum(dim=(1, 2))).abs() <= rel * p.sum(dim=(1, 2))).all()
            order = cache.order[page, :, off].t()
            assert (order == torch.arange(prompt, device="cuda")).all()
            before.append(cache.weights[page, :, off].t().cpu().numpy())
        found.append(before)
        evict(cache, *args, **kw)
        for b in range(B):
            page, off = slots(cache, b, budget)
            for h in range(KV):
                want = oc.evict(before[b][h], list(range(prompt)), prompt, budget, recent)
                assert cache.order[page, h, off].tolist() == want, (b, h)
    monkeypatch.setattr(m, "mosaic_cache_append", keep_queries)
    monkeypatch.setattr(m, "mosaic_cache_evict", check_weights)
    got, kept = torch.empty_like(x), {}
    got[:, :prompt] = d.prompt(x[:, :prompt].reshape(B * prompt, H)).view(B, prompt, H)
    assert len(found) == CFG["layers"] and d.held == budget and d.seen == prompt
    if sharp > 1:                                   # the heads do not agree on what to keep
        assert any(len({tuple(c.order[slots(c, b, budget)[0], h, slots(c, b, budget)[1]].tolist())
                        for b in range(B) for h in range(KV)}) > 1 for c in d.caches)
        return
    monkeypatch.undo()
    for t in range(prompt, S):
        for l, c in enumerate(d.caches):
            for b in range(B):
                page, off = slots(c, b, budget)
                for h in range(KV):
                    kept[l, b, h, t] = torch.cat([c.order[page, h, off].long(), torch.tensor([t], device="cuda")])
        got[:, t] = d.step(x[:, t].contiguous())
    want = reference(weights, x, CFG, table, (32,), lambda l, b, h, t: kept.get((l, b, h, t)))
    e = dec.error_metrics(got, want)
    assert e["rel_l2"] < 3e-5, e
