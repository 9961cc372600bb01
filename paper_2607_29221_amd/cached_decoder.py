"""Token-by-token decoding of the decoder stack (decoder.py) with the keys and
values of all tokens kept by the trusted client.

Every linear layer is whatever the caller passes (Pi_Sec-Linear calls of a
SecureDecoder, or plain products); attention and its cache are the client's
own operators: mosaic_cache_append rotates and stores a layer's new queries,
keys and values, mosaic_cache_attend attends from one new token per sequence,
and with a budget mosaic_cache_evict keeps, per layer and key/value head, the
latest tokens and those that got most attention weight so far.

A prompt goes through all layers at once. Its attention is float32 torch
operations, as in decoder.attention (a prompt's products with all its own
tokens are no decoding step); with a budget its weights are added up too, so
that the first eviction already knows what the prompt attended to.
"""
from __future__ import annotations

import math
from typing import Callable, List, Optional, Sequence, Tuple

import torch

from . import mosaic as m
from .decoder import SecureDecoder, rms_norm

Linear = Callable[[int, str, torch.Tensor], torch.Tensor]


def secure_linears(decoder: SecureDecoder) -> Linear:
    """The linear layers of a SecureDecoder, each call under a fresh id."""
    def linear(layer: int, name: str, x: torch.Tensor) -> torch.Tensor:
        decoder.calls += 1
        return decoder.layers[layer][name](x, call_id=decoder.calls)
    return linear


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Causal attention of one sequence's prompt in float32: q (tokens x heads
    x dim), k and v (kv_heads x tokens x dim). Returns the outputs (tokens x
    heads * dim) and the weight that each token got (kv_heads x tokens)."""
    n, heads, dim = q.shape
    kv = k.shape[0]
    s = torch.matmul(q.transpose(0, 1).reshape(kv, heads // kv * n, dim), k.transpose(1, 2).contiguous())
    s = s.reshape(kv, heads // kv, n, n) * (1.0 / math.sqrt(dim))
    s.masked_fill_(torch.ones((n, n), dtype=torch.bool, device=q.device).triu_(1), float("-inf"))
    p = torch.softmax(s, dim=-1)
    out = torch.matmul(p.reshape(kv, heads // kv * n, n), v).reshape(heads, n, dim)
    return out.transpose(0, 1).reshape(n, heads * dim), p.sum(dim=(1, 2))


class CachedDecoder:
    """Decoding with a cache of ``max_len`` slots per sequence and layer.

    ``dtype`` is the cache's (activations are float32). ``table`` and
    ``sections`` give rotary positions (mosaic.Rotary; None: none, as in
    decoder.py); calls without ``positions`` turn a token by its number, up to
    the table's last row. ``budget``: tokens that a head keeps after every call, the
    ``recent`` latest among them; None keeps all. Where the slots are as many
    as the budget the caches get room for the token that comes on top; a
    larger budget is never reached, and a full cache ends the decode.

    A call that raises (a linear layer of a server that cannot be reached, or
    whose products fail their check) leaves the decoder as it was, and can be
    made again; with a budget, a step that fails after its first layer's q|k|v
    product cannot be undone, and further calls are refused."""

    def __init__(self, linear: Linear, layers: int, cfg: dict, max_len: int, dtype=torch.float32, page_size: int = 64,
                 budget: Optional[int] = None, recent: int = 0, table: Optional[torch.Tensor] = None,
                 sections: Optional[Sequence[int]] = None, interleaved: bool = False, device="cuda"):
        if budget is not None and budget < 1:
            raise ValueError("a budget keeps at least one token")
        if budget is not None and not 0 <= recent <= budget:
            raise ValueError("recent must lie between 0 and the budget")
        if (table is None) != (sections is None):
            raise ValueError("rotary positions need a table and sections")
        if budget is not None and budget == -(-max_len // page_size) * page_size:
            max_len = budget + 1             # the next token comes before the one that it replaces goes
        self.linear, self.cfg, self.budget, self.recent = linear, cfg, budget, recent
        self.table, self.sections, self.interleaved = table, sections, interleaved
        self.caches: List[m.KVCache] = [
            m.KVCache.empty(cfg["batch"], max_len, cfg["kv_heads"], cfg["head_dim"], dtype, page_size,
                            evicts=budget is not None, device=device) for _ in range(layers)]
        self.held = self.seen = 0            # tokens per sequence, the same in every layer; evicted ones among the seen
        self.torn = False                    # a call failed and left tokens in some layers only

    def _check_places(self, tokens: int, positions) -> None:
        if self.table is not None and positions is None and self.seen + tokens > self.table.shape[0]:
            raise ValueError(f"the rotary table has {self.table.shape[0]} places, {self.seen} tokens were seen before "
                             f"these {tokens}")

    def _append(self, cache: m.KVCache, qkv: torch.Tensor, starts, positions) -> torch.Tensor:
        cfg = self.cfg
        q = torch.empty((qkv.shape[0], cfg["heads"] * cfg["head_dim"]), dtype=qkv.dtype, device=qkv.device)
        rotary = None if self.table is None else m.Rotary(self.table, self.sections, positions, self.interleaved)
        m.mosaic_cache_append(cache, qkv, cfg["heads"], q, starts=starts, rotary=rotary)
        return q

    def _layers(self, h: torch.Tensor, tokens: int, attend) -> torch.Tensor:
        """All layers over ``tokens`` new tokens of each sequence;
        attend(cache, qkv, held) appends them, which makes ``held`` in all. The
        counts advance once the last layer is through."""
        F, held, started = self.cfg["ffn"], self.held + tokens, False
        try:
            for i, cache in enumerate(self.caches):
                qkv = self.linear(i, "qkv", rms_norm(h).contiguous())
                started = True
                h = h + self.linear(i, "o", attend(cache, qkv, held))
                gu = self.linear(i, "gate_up", rms_norm(h).contiguous())
                h = h + self.linear(i, "down", (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]).contiguous())
                if self.budget is not None and held > self.budget:
                    m.mosaic_cache_evict(cache, self.budget, self.recent, max_len=held)
        except BaseException:
            if started:
                self._take_back()
            raise
        self.held = held if self.budget is None else min(held, self.budget)
        self.seen += tokens
        return h

    def _take_back(self) -> None:
        """The caches as before a call that failed in the middle of the layers.
        What lies behind the tokens held has no meaning; the weights that the
        call added to theirs, and what it evicted, cannot be undone."""
        self.torn = self.budget is not None and self.held > 0
        if not self.torn:
            for cache in self.caches:
                cache.state[0].fill_(self.held)
                cache.state[1].fill_(self.seen)

    def _check_whole(self) -> None:
        if self.torn:
            raise RuntimeError("an earlier step failed in the middle of the layers, after it had changed weights and "
                               "tokens of some: this decoder's caches cannot be used any more")

    def prompt(self, x: torch.Tensor, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Hidden states (batch * seq x hidden) of a prompt, sequence after
        sequence, into an empty cache; ``positions``: axes x rows."""
        self._check_whole()
        B = self.cfg["batch"]
        n = x.shape[0] // B
        if self.held != 0 or n * B != x.shape[0]:
            raise ValueError("a prompt needs an empty cache, and sequences of one length")
        if n > self.caches[0].slots:
            raise ValueError(f"a prompt of {n} tokens does not fit {self.caches[0].slots} slots")
        self._check_places(n, positions)
        starts = torch.arange(B + 1, dtype=torch.int32, device=x.device) * n

        def attend(cache: m.KVCache, qkv: torch.Tensor, held: int) -> torch.Tensor:
            q = self._append(cache, qkv, starts, positions)
            heads, dim, page = self.cfg["heads"], self.cfg["head_dim"], cache.k.shape[2]
            out = torch.empty_like(q)
            slot = torch.arange(n, device=x.device)
            for b in range(B):               # one sequence at a time bounds the score memory
                where, off = cache.block_table[b].long()[slot // page], slot % page
                k, v = (t[where, :, off].float().transpose(0, 1).contiguous() for t in (cache.k, cache.v))
                out[b * n: (b + 1) * n], got = prompt_attention(q[b * n: (b + 1) * n].view(n, heads, dim), k, v)
                if cache.weights is not None:
                    cache.weights[where, :, off] += got.t()
            return out

        return self._layers(x, n, attend)

    def step(self, x: torch.Tensor, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Hidden states of the next token (batch x hidden; positions: axes x
        batch), one per sequence."""
        self._check_whole()
        if x.shape[0] != self.cfg["batch"]:
            raise ValueError("a step takes one token per sequence")
        if self.held >= self.caches[0].slots:
            raise ValueError(f"no slot is free: {self.held} tokens are held")
        self._check_places(1, positions)

        def attend(cache: m.KVCache, qkv: torch.Tensor, held: int) -> torch.Tensor:
            q = self._append(cache, qkv, None, positions)
            out = torch.empty_like(q)
            m.mosaic_cache_attend(cache, q, self.cfg["heads"], out, max_len=held,
                                  accumulate=cache.weights is not None)
            return out

        return self._layers(x, 1, attend)
