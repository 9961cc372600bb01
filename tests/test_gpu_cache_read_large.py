"""Cached tokens as rows, many at a time: outputs that pass by the caches, several
rows for a group of threads, and a last workgroup that is not full."""
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests import cache_util as cu
from tests import e2m1_util as eu
from tests.cache_util import DT, same_bits, seeded
from tests.test_gpu_cache_attend_e2m1_forms import random_cache

pytestmark = pytest.mark.gpu


def check(c, values, lengths, out, gap=0):
    """values: what the cache holds of k and v, (tokens of all sequences x kv_heads * dim) each."""
    rows, width = values[0].shape
    ko, vo = (torch.full((rows + 1, width + gap), 7.0, dtype=DT[out], device="cuda") for _ in range(2))
    starts = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")
    m.mosaic_cache_read(c, ko[:rows, :width], vo[:rows, :width], starts=starts)
    for got, want in zip((ko, vo), values):
        assert same_bits(got[:rows, :width], want.to(DT[out])) and (got[rows:] == 7).all() and (got[:, width:] == 7).all()


def held(c, lengths, unpack):
    res = []
    for t in (c.k, c.v):
        parts = []
        for b, n in enumerate(lengths):
            p, o = eu.where(c, b, 0, n)
            parts.append(unpack(t[p, :, o]).reshape(n, t.shape[1] * (t.shape[3] if c.head_dim is None else c.head_dim)))
        res.append(torch.cat(parts))
    return res


# rows x heads x dim: streamed with four rows of a group, streamed with groups of 8 lanes and two rows, not streamed with three
SHAPES = (((8192, 3), 8, 128, "f32"), ((70001,), 1, 64, "bf16"), ((60000, 0, 40007), 1, 64, "f16"), ((100003,), 1, 8, "f32"),
          ((12289, 1), 2, 72, "bf16"), ((3000, 2501), 4, 256, "f32"))


@pytest.mark.parametrize("lengths,kv,dim,out", SHAPES, ids=lambda v: str(v).replace(" ", ""))
def test_rows_of_4_bits(lengths, kv, dim, out):
    c = random_cache(lengths, kv, dim, 64, 5)
    values = held(c, lengths, lambda t: torch.from_numpy(oc.unpack_e2m1(t.cpu().numpy(), dim)).cuda())
    check(c, values, lengths, out, gap=8 if dim == 72 else 0)


@pytest.mark.parametrize("lengths,kv,dim", (((8192, 3), 8, 128), ((70001,), 1, 64), ((100003,), 1, 16)))
@pytest.mark.parametrize("out,cache", (("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f16")))
def test_rows_of_16_and_32_bits(lengths, kv, dim, out, cache):
    c = cu.make_cache([0] * len(lengths), kv, dim, 64, cache, 6, room=max(lengths))
    c.state.copy_(torch.tensor([lengths] * 2, dtype=torch.int32))
    g = seeded(7)
    for b, n in enumerate(lengths):
        p, o = eu.where(c, b, 0, n)
        for t in (c.k, c.v):
            t[p, :, o] = torch.randn((n, kv, dim), generator=g, device="cuda").to(DT[cache])
    check(c, held(c, lengths, lambda t: t), lengths, out)
