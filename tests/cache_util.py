"""Paged caches for the tests: random tables, memory that holds no token filled
with NaN, and what the pages hold as plain arrays."""
import numpy as np
import torch

from paper_2607_29221_amd import mosaic as m

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half the spacing of the type relative to a value, 2^-(explicit bits + 1), and half the smallest step of f16
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
# (activations, cache): all that the entry points take
TYPES = (("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16"))


def seeded(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make_cache(lengths, kv_heads, dim, page, cache, seed, layout="heads", room=0, evicts=False, gap=0, seen=None,
               junk=float("nan")):
    """Sequences of the given lengths, with ``room`` more slots at least; their
    pages scattered; every other element of the memory holds ``junk``."""
    g = seeded(seed)
    B = len(lengths)
    blocks = max(1, -(-(max(lengths) + room) // page)) if B else 1
    pages = B * blocks + 3
    shape = (pages, kv_heads, page, dim + gap) if layout == "heads" else (pages, page, kv_heads, dim + gap)
    def memory():
        t = torch.full(shape, junk, dtype=DT[cache], device="cuda")
        return (t if layout == "heads" else t.transpose(1, 2))[..., :dim]
    c = m.KVCache(memory(), memory(), torch.randperm(pages, generator=g, device="cuda")[: B * blocks]
                  .to(torch.int32).reshape(B, blocks),
                  torch.tensor([list(lengths), list(lengths if seen is None else seen)], dtype=torch.int32,
                               device="cuda"))
    if evicts:
        c.weights = torch.full((pages, kv_heads, page), junk, device="cuda")
        c.order = torch.full((pages, kv_heads, page), -7, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lengths):
        for name in ("k", "v"):
            x = torch.randn((kv_heads, n, dim), generator=g, device="cuda").to(DT[cache])
            put(c, name, b, x)
        if evicts:
            put(c, "weights", b, torch.rand((kv_heads, n), generator=g, device="cuda"))
            put(c, "order", b, torch.arange(n, device="cuda", dtype=torch.int32).expand(kv_heads, n))
    return c


def _where(c, b, n):
    page = c.k.shape[2]
    i = torch.arange(n, device="cuda")
    return c.block_table[b].long()[i // page], i % page


def put(c, name, b, x):
    """Writes rows (kv_heads x tokens ...) into the first slots of sequence b."""
    if x.shape[1]:
        p, o = _where(c, b, x.shape[1])
        getattr(c, name)[p, :, o] = x.transpose(0, 1)


def get(c, name, b, n):
    """The first n slots of sequence b (kv_heads x n ...), in float64 or int."""
    t = getattr(c, name)
    p, o = _where(c, b, n)
    x = t[p, :, o].transpose(0, 1)
    return (x.double() if x.is_floating_point() else x).cpu().numpy()


def clone(c):
    return m.KVCache(*(None if t is None else t.clone(memory_format=torch.preserve_format)
                       for t in (c.k, c.v, c.block_table, c.state, c.weights, c.order)))


def same_bits(a, b):
    """Equal, NaN included."""
    return torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0)) \
        if a.is_floating_point() else torch.equal(a, b)


def f64(t):
    return t.double().cpu().numpy()
