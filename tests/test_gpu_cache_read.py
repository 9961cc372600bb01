"""Cached tokens as rows: what the pages hold, converted once; zeros where a slot
holds no token; nothing else written."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests import cache_util as cu
from tests import e2m1_util as eu
from tests.cache_util import DT, TYPES, same_bits

pytestmark = pytest.mark.gpu


def expected(c, util, b, first, count, out):
    """Keys and values (count x kv_heads * dim) of slots of sequence b as the call gives them."""
    dim = c.k.shape[3] if c.head_dim is None else c.head_dim
    KV, n = c.k.shape[1], max(0, min(int(c.state[0, b]), c.slots))
    res = []
    for name in ("k", "v"):
        rows = torch.zeros((count, KV, dim), dtype=torch.float64)
        held = torch.from_numpy(util.get(c, name, b, n)).double()          # kv_heads x n x dim
        for i in range(count):
            s = first + i
            if 0 <= s < n and 0 <= int(c.block_table[b, s // c.k.shape[2]]) < c.k.shape[0]:
                rows[i] = held[:, s]
        res.append(rows.reshape(count, KV * dim).to(DT[out]))
    return res


def read(c, counts, out, firsts=None, starts=True, gap=0):
    dim = c.k.shape[3] if c.head_dim is None else c.head_dim
    rows, width = sum(counts), c.k.shape[1] * dim
    ko, vo = (torch.full((rows + 2, width + gap), 7.0, dtype=DT[out], device="cuda") for _ in range(2))
    s = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda") if starts else None
    f = None if firsts is None else torch.tensor(firsts, dtype=torch.int32, device="cuda")
    m.mosaic_cache_read(c, ko[:rows, :width], vo[:rows, :width], starts=s, first=f)
    assert (ko[rows:] == 7).all() and (vo[rows:] == 7).all() and (ko[:, width:] == 7).all() and (vo[:, width:] == 7).all()
    return ko[:rows, :width], vo[:rows, :width]


def check(c, util, counts, out, firsts=None, starts=True, gap=0):
    ko, vo = read(c, counts, out, firsts, starts, gap)
    t = 0
    for b, n in enumerate(counts):
        for got, want in zip((ko, vo), expected(c, util, b, 0 if firsts is None else firsts[b], n, out)):
            assert same_bits(got[t: t + n].cpu(), want), b
        t += n


@pytest.mark.parametrize("dim", (8, 40, 64, 80, 128, 256))
@pytest.mark.parametrize("out", eu.ACTS)
def test_rows_of_4_bits(dim, out):
    lengths = (0, 1, 40, 17, 100)
    c = eu.make_cache(lengths, 3, dim, 16, 5, layout="tokens" if dim == 80 else "heads", gap=16 if dim == 64 else 0)
    check(c, eu, lengths, out, gap=8 if dim == 40 else 0)
    check(c, eu, (1, 0, 13, 3, 64), out, firsts=(0, 5, 30, 14, 36))
    check(c, eu, (1,) * 5, out, firsts=(0, 0, 39, 3, 99), starts=False)


@pytest.mark.parametrize("out,cache", TYPES)
def test_rows_of_16_and_32_bits(out, cache):
    lengths = (0, 1, 40, 17)
    c = cu.make_cache(lengths, 2, 80, 16, cache, 6, layout="tokens")
    check(c, cu, lengths, out)
    check(c, cu, (2, 0, 11, 3), out, firsts=(0, 1, 30, 14))


def test_slots_without_tokens():
    """Before the first, behind the last, on pages that are not there, of
    negative lengths and lengths beyond the table."""
    c = eu.make_cache((20, 33, 5, 16), 2, 64, 16, 7)
    c.block_table[1, 0], c.block_table[1, 2] = -1, c.k.shape[0]
    c.state[0, 2], c.state[0, 3] = -3, 1000
    check(c, eu, (40, 60, 8, 60), "f32", firsts=(-10, -5, 0, 0))
    far = (2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1)
    ko, vo = read(c, (3, 2, 2, 2), "f32", firsts=far)
    assert not ko.any() and not vo.any()


def test_nan_scales():
    c = eu.make_cache((4,), 1, 16, 16, 8)
    p, o = eu.where(c, 0, 2, 1)
    c.k[p, :, o, 8] = 255
    ko, vo = read(c, (4,), "bf16")
    assert torch.isnan(ko[2, :8]).all() and torch.isnan(ko).sum() == 8 and not torch.isnan(vo).any()


def test_a_prompt_and_many_sequences():
    lengths = [int(n) for n in np.random.default_rng(3).integers(0, 40, 300)]
    c = eu.make_cache(lengths, 2, 64, 16, 9)
    check(c, eu, lengths, "f32")
    c = eu.make_cache((3000,), 2, 64, 64, 10)
    check(c, eu, (3000,), "bf16")


@pytest.mark.parametrize("dim,out", ((8, "f16"), (8, "f32"), (16, "f32"), (24, "bf16")))
def test_short_rows(dim, out):
    """Rows of a few 16-byte pieces, many of which a workgroup takes."""
    lengths = (2500, 0, 1, 300)
    c = eu.make_cache(lengths, 1, dim, 64, 15)
    check(c, eu, lengths, out)
    check(c, eu, (7, 0, 3, 290), out, firsts=(2490, 3, 0, 9))


def test_shared_table_stream_and_graph():
    """A table row that all sequences share, on a side stream, captured and replayed."""
    c = eu.make_cache((50,), 2, 64, 16, 11)
    shared = m.KVCache(c.k, c.v, c.block_table.expand(3, -1), torch.tensor([[50, 7, 20]] * 2, dtype=torch.int32, device="cuda"),
                       head_dim=64)
    first = torch.tensor([40, 0, 10], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 10, 17, 27], dtype=torch.int32, device="cuda")
    ko, vo = (torch.zeros((27, 128), device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.mosaic_cache_read(shared, ko, vo, starts=starts, first=first)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    kg, vg = torch.zeros_like(ko), torch.zeros_like(vo)
    with torch.cuda.graph(graph):
        m.mosaic_cache_read(shared, kg, vg, starts=starts, first=first)
    for _ in range(3):
        kg.zero_(), vg.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kg, ko) and torch.equal(vg, vo)
    whole = torch.from_numpy(oc.unpack_e2m1(eu.rows_of(c, "k", 0, 0, 50), 64)).float().transpose(0, 1).reshape(50, 128)
    assert torch.equal(ko.cpu(), torch.cat([whole[40:], whole[:7], whole[10:20]]))


def test_no_rows():
    c = eu.make_cache((4, 2), 1, 16, 16, 12)
    m.mosaic_cache_read(c, torch.empty((0, 16), device="cuda"), torch.empty((0, 16), device="cuda"),
                        starts=torch.zeros(3, dtype=torch.int32, device="cuda"))


def test_refusals():
    c = eu.make_cache((3, 4), 2, 64, 16, 13)
    ko, vo = (torch.zeros((2, 128), device="cuda") for _ in range(2))
    m.mosaic_cache_read(c, ko, vo)
    both = torch.zeros((2, 256), device="cuda")
    for k, v in ((ko[:1], vo[:1]), (both[:, :128], both[:, 64: 192])):     # rows without starts; one over the other
        with pytest.raises(m.MosaicError) as e:
            m.mosaic_cache_read(c, k, v)
        assert e.value.status == m.STATUS_INVALID_ARG
    inside = c.k.view(torch.uint8).flatten()[: 2 * 128 * 4].view(torch.float32).reshape(2, 128)
    with pytest.raises(m.MosaicError):
        m.mosaic_cache_read(c, inside, vo)
    plain = cu.make_cache((3, 4), 2, 64, 16, "bf16", 14)
    for cache, k, v, kw in ((c, ko[:, :64], vo, {}), (c, ko, vo.half(), {}), (c, ko.cpu(), vo, {}), (c, ko.double(), vo.double(), {}),
                            (plain, ko.half(), vo.half(), {}), (c, ko, vo[:1], {}),
                            (c, ko, vo, dict(starts=torch.zeros(2, dtype=torch.int32, device="cuda"))),
                            (c, ko, vo, dict(first=torch.zeros(2, dtype=torch.int64, device="cuda"))),
                            (c, ko, vo, dict(first=torch.zeros(3, dtype=torch.int32, device="cuda")))):
        with pytest.raises(ValueError):
            m.mosaic_cache_read(cache, k, v, **kw)
