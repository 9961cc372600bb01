"""Decoding with a cache, layer by layer through the client's operators: the same
hidden states as the forward pass over the whole sequence (decoder.py), with
rotary positions as a plain computation in float64, and with a budget as that
computation over the tokens which the cache says it still holds."""
import math

import pytest
import torch

from paper_2607_29221_amd import decoder as dec
from paper_2607_29221_amd import mosaic as m
from paper_2607_29221_amd.cached_decoder import CachedDecoder, prompt_attention, secure_linears
from synthetic_inputs import (DECODER_LINEARS, DECODER_SEED, PARAMS_D1_SMALL_R128, decoder_input, decoder_weight)

CFG = dict(hidden=256, heads=4, kv_heads=2, head_dim=64, ffn=512, layers=2, batch=2, seq=40)
PROTOCOL_SEED = 0x6D6F736169630000 | DECODER_SEED


@pytest.fixture(autouse=True)
def _no_reduced_precision():
    prev = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = prev


def stack(cfg=CFG):
    dev = torch.device("cuda", 0)
    weights = [{n: decoder_weight(l, n, dev, cfg) for n in DECODER_LINEARS} for l in range(cfg["layers"])]
    x = decoder_input(dev, cfg).view(cfg["batch"], cfg["seq"], cfg["hidden"])
    return weights, x


def plain(weights):
    return lambda layer, name, a: torch.nn.functional.linear(a, weights[layer][name])


def run(decoder, x, prompt):
    """Hidden states of all tokens (batch x seq x hidden): a prompt, then steps."""
    B, S, H = x.shape
    out = torch.empty_like(x)
    out[:, :prompt] = decoder.prompt(x[:, :prompt].reshape(B * prompt, H)).view(B, prompt, H)
    for t in range(prompt, S):
        out[:, t] = decoder.step(x[:, t].contiguous())
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("prompt", (1, 17, 39))
def test_steps_equal_the_whole_forward(prompt):
    """Float32 throughout: two layers of products of at most 512 terms, each off
    by its rounding in either order of summation (512 u = 3e-5 at worst)."""
    weights, x = stack()
    want = dec.plaintext_forward(x.reshape(-1, CFG["hidden"]), weights, CFG)[-1].view_as(x)
    got = run(CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], page_size=16), x, prompt)
    e = dec.error_metrics(got, want)
    assert e["rel_l2"] < 3e-5, e


@pytest.mark.gpu
def test_cache_in_16_bits():
    """Keys and values rounded to bf16 (2^-9 of each on average): the hidden
    state moves by less than one rounding of everything."""
    weights, x = stack()
    want = dec.plaintext_forward(x.reshape(-1, CFG["hidden"]), weights, CFG)[-1].view_as(x)
    for dtype, bound in ((torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)):
        got = run(CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], dtype=dtype, page_size=16), x, 10)
        e = dec.error_metrics(got, want)
        assert e["rel_l2"] < bound, (dtype, e)


@pytest.mark.gpu
def test_secure_steps_track_plaintext():
    """The linear layers behind Pi_Sec-Linear, one token at a time: the error of
    the masked products, as for the whole forward (tests/test_gpu_decoder.py)."""
    weights, x = stack()
    sd = dec.SecureDecoder(weights, CFG, PARAMS_D1_SMALL_R128, PROTOCOL_SEED)
    want = dec.plaintext_forward(x.reshape(-1, CFG["hidden"]), weights, CFG)[-1].view_as(x)
    got = run(CachedDecoder(secure_linears(sd), CFG["layers"], CFG, CFG["seq"], page_size=16, budget=64, recent=4), x, 30)
    e = dec.error_metrics(got, want)
    assert e["rel_l2"] < 0.25 and e["cosine"] > 0.97, e
    assert sd.calls == 2 * 4 * (1 + 10)


def reference(weights, x, cfg, table, sections, held=None):
    """All tokens in float64 with rotary positions (pairs j and P + j, places on
    all axes alike); held(layer, b, h, t): the tokens that token t attends to."""
    B, S, H = x.shape
    heads, kv, D, F = cfg["heads"], cfg["kv_heads"], cfg["head_dim"], cfg["ffn"]
    P = sum(sections)
    cos, sin = table[:S, :P].double(), table[:S, P:].double()
    def norm(a):
        return a / torch.sqrt((a * a).mean(-1, keepdim=True) + 1e-5)
    def turn(a):                                     # (B, S, heads, D)
        u, v = a[..., :P], a[..., P: 2 * P]
        c, s = cos[:, None, :], sin[:, None, :]
        return torch.cat([u * c - v * s, v * c + u * s, a[..., 2 * P:]], -1)
    h = x.double()
    for l, layer in enumerate(weights):
        W = {n: w.double() for n, w in layer.items()}
        qkv = norm(h) @ W["qkv"].t()
        q = turn(qkv[..., : heads * D].reshape(B, S, heads, D))
        k = turn(qkv[..., heads * D: (heads + kv) * D].reshape(B, S, kv, D))
        v = qkv[..., (heads + kv) * D:].reshape(B, S, kv, D)
        a = torch.empty_like(q)
        for b in range(B):
            for g in range(heads):
                j = g // (heads // kv)
                s = q[b, :, g] @ k[b, :, j].t() / math.sqrt(D)
                mask = torch.ones((S, S), dtype=torch.bool, device=x.device).tril()
                if held is not None:
                    for t in range(S):
                        only = held(l, b, j, t)
                        if only is not None:
                            mask[t] = False
                            mask[t, only] = True
                a[b, :, g] = torch.softmax(s.masked_fill(~mask, float("-inf")), -1) @ v[b, :, j]
        h = h + a.reshape(B, S, heads * D) @ W["o"].t()
        gu = norm(h) @ W["gate_up"].t()
        h = h + (torch.nn.functional.silu(gu[..., :F]) * gu[..., F:]) @ W["down"].t()
    return h


@pytest.mark.gpu
@pytest.mark.parametrize("sections", ((32,), (4, 10, 6)))
def test_rotary_positions(sections):
    weights, x = stack()
    table = m.Rotary.frequencies(64, sum(sections))
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], page_size=16, table=table, sections=sections)
    e = dec.error_metrics(run(d, x, 12), reference(weights, x, CFG, table, sections))
    assert e["rel_l2"] < 3e-5, e


@pytest.mark.gpu
def test_budget():
    """Tokens go once a head holds more than 16; what the layers compute is
    attention over the rest, positions and all."""
    weights, x = stack()
    sections, budget, recent, prompt = (32,), 16, 5, 12
    table = m.Rotary.frequencies(64, 32)
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], page_size=16, table=table, sections=sections,
                      budget=budget, recent=recent)
    B, S, H = x.shape
    kept, got = {}, torch.empty_like(x)
    got[:, :prompt] = d.prompt(x[:, :prompt].reshape(B * prompt, H)).view(B, prompt, H)
    for t in range(prompt, S):
        for l, c in enumerate(d.caches):
            n = min(t, budget)
            assert c.state.tolist() == [[n] * B, [t] * B]
            for b in range(B):
                page, off = c.block_table[b].long()[torch.arange(n) // 16], torch.arange(n, device="cuda") % 16
                for h in range(CFG["kv_heads"]):
                    order = c.order[page, h, off].long()
                    assert len(set(order.tolist())) == n and set(range(t - min(recent, n), t)) <= set(order.tolist())
                    kept[l, b, h, t] = torch.cat([order, torch.tensor([t], device="cuda")])
        got[:, t] = d.step(x[:, t].contiguous())
    want = reference(weights, x, CFG, table, sections, lambda l, b, h, t: kept.get((l, b, h, t)))
    e = dec.error_metrics(got, want)
    assert e["rel_l2"] < 3e-5, e


@pytest.mark.gpu
def test_weights_of_prompt_and_steps():
    """What eviction goes by: every query's weights sum to one, so a head's
    add up to the queries of its group."""
    weights, x = stack()
    d = CachedDecoder(plain(weights), CFG["layers"], CFG, CFG["seq"], page_size=16, budget=1000)
    run(d, x, 25)
    c = d.caches[1]
    n = CFG["seq"]
    for b in range(CFG["batch"]):
        page, off = c.block_table[b].long()[torch.arange(n) // 16], torch.arange(n, device="cuda") % 16
        total = c.weights[page, :, off].double().sum(0)
        assert ((total - 2 * n).abs() < 2 * n * n * 2.0 ** -24 * 4).all(), total


@pytest.mark.gpu
def test_what_a_cached_decoder_refuses():
    weights, x = stack()
    lin = plain(weights)
    with pytest.raises(ValueError):
        CachedDecoder(lin, 2, CFG, 16, budget=4, recent=5)
    with pytest.raises(ValueError):
        CachedDecoder(lin, 2, CFG, 16, sections=[32])
    d = CachedDecoder(lin, 2, CFG, 16, page_size=16)
    with pytest.raises(ValueError):
        d.prompt(x[:, :17].reshape(34, -1))
    with pytest.raises(ValueError):
        d.prompt(x[:, :3].reshape(6, -1)[:5])
    d.prompt(x[:, :16].reshape(32, -1))
    with pytest.raises(ValueError):
        d.step(x[:, 16].contiguous())
    with pytest.raises(ValueError):
        d.prompt(x[:, :2].reshape(4, -1))


def test_prompt_attention_on_the_host():
    """Against the attention of the whole-sequence decoder, without a GPU."""
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((9, 8 * 16), generator=g)
    cfg = dict(batch=1, seq=9, heads=4, kv_heads=2, head_dim=16)
    want = dec.attention(qkv, cfg)
    out, w = prompt_attention(qkv[:, :64].view(9, 4, 16), qkv[:, 64:96].view(9, 2, 16).transpose(0, 1),
                              qkv[:, 96:].view(9, 2, 16).transpose(0, 1))
    assert torch.allclose(out, want, atol=1e-6)
    assert torch.allclose(w.sum(1), torch.full((2,), 18.0), atol=1e-4)
