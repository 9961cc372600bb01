"""Paged caches in 4 bits for the tests: random tables, memory that holds no token
filled with bytes of 255 (NaN), and what the pages hold as plain arrays."""
import numpy as np
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests.cache_util import seeded

ACTS = ("f32", "bf16", "f16")


def make_cache(lengths, kv_heads, dim, page, seed, layout="heads", room=0, evicts=False, gap=0, seen=None, scale=1.0):
    """Sequences of the given lengths, with ``room`` more slots at least; their
    pages scattered; ``gap`` bytes between rows."""
    g = seeded(seed)
    B = len(lengths)
    blocks = max(1, -(-(max(lengths) + room) // page)) if B else 1
    pages = B * blocks + 3
    width = m.KVCache.row_bytes(dim)
    shape = (pages, kv_heads, page, width + gap) if layout == "heads" else (pages, page, kv_heads, width + gap)

    def memory():
        t = torch.full(shape, 255, dtype=torch.uint8, device="cuda")
        return (t if layout == "heads" else t.transpose(1, 2))[..., :width]
    c = m.KVCache(memory(), memory(), torch.randperm(pages, generator=g, device="cuda")[: B * blocks]
                  .to(torch.int32).reshape(B, blocks),
                  torch.tensor([list(lengths), list(lengths if seen is None else seen)], dtype=torch.int32,
                               device="cuda"), head_dim=dim)
    if evicts:
        c.weights = torch.full((pages, kv_heads, page), float("nan"), device="cuda")
        c.order = torch.full((pages, kv_heads, page), -7, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lengths):
        for name in ("k", "v"):
            put(c, name, b, torch.randn((kv_heads, n, dim), generator=g, device="cuda") * scale)
        if evicts and n:
            p, o = where(c, b, 0, n)
            c.weights[p, :, o] = torch.rand((n, kv_heads), generator=g, device="cuda")
            c.order[p, :, o] = torch.arange(n, device="cuda", dtype=torch.int32)[:, None].expand(n, kv_heads)
    return c


def where(c, b, first, count):
    """Page and place of slots; entries of the table that are no page are some page
    (torch must not index with them)."""
    i = first + torch.arange(count, device="cuda")
    page = c.k.shape[2]
    assert first >= 0 and first + count <= c.slots
    return c.block_table[b].long().clamp(0, c.k.shape[0] - 1)[i // page], i % page


def put(c, name, b, x, first=0):
    """Writes values (kv_heads x tokens x dim) from slot ``first`` of sequence b on."""
    if x.shape[1]:
        rows = torch.from_numpy(oc.pack_e2m1(*oc.to_e2m1(x.double().cpu().numpy()))).cuda()
        p, o = where(c, b, first, x.shape[1])
        getattr(c, name)[p, :, o] = rows.transpose(0, 1)


def rows_of(c, name, b, first, count):
    """Bytes of slots (kv_heads x count x row)."""
    p, o = where(c, b, first, count)
    return getattr(c, name)[p, :, o].transpose(0, 1).cpu().numpy()


def get(c, name, b, n):
    """The first n slots of sequence b (kv_heads x n ...), in float64 or int."""
    if name in ("k", "v"):
        return oc.unpack_e2m1(rows_of(c, name, b, 0, n), c.head_dim)
    p, o = where(c, b, 0, n)
    x = getattr(c, name)[p, :, o].transpose(0, 1)
    return (x.double() if x.is_floating_point() else x).cpu().numpy()


def clone(c):
    return m.KVCache(*(None if t is None else t.clone(memory_format=torch.preserve_format)
                       for t in (c.k, c.v, c.block_table, c.state, c.weights, c.order)), head_dim=c.head_dim)
