"""Scores beyond the range of float32 over a cache in 4 bits: finite queries and
keys whose products add up to less than -2^128 make a score of -inf, which is no
weight; the other tokens' outputs and weights are as without them.

The tokens in reach: tolerance of test_gpu_cache_attend_e2m1.py, from them alone
(a weight of exactly 0 adds nothing to any sum)."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests import e2m1_util as eu
from tests.cache_util import DT, TINY, UNIT, f64, seeded
from tests.test_gpu_cache_attend_e2m1 import PARTS, U

pytestmark = pytest.mark.gpu

# the forms of the kernel: heads side by side, one and several blocks of heads, whole and padded head dimensions
SHAPES = ((4, 1, 64), (7, 1, 64), (8, 2, 128), (8, 1, 128), (3, 3, 256), (6, 1, 256), (16, 1, 128), (6, 2, 80), (40, 1, 128),
          (20, 1, 64), (20, 1, 256), (48, 1, 200))
# large elements of queries and keys by the activations' type: their products are 2^136 and more, those of what
# 8 bits leave of a query's element (0.375 * 2^-7 of its power of two, as it is made here) 2^127 and more each
LARGE = {"f32": (2.0 ** 126, 2.0 ** 10), "bf16": (2.0 ** 126, 2.0 ** 10), "f16": (2.0 ** 15, 2.0 ** 121)}


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim", SHAPES)
@pytest.mark.parametrize("part", ("against", "along", "mixed"))
def test_scores_beyond_the_range(act, heads, kv, dim, part):
    """``part``: whether what 8 bits leave of a query's elements lies against their
    own signs, along with them, or either."""
    lengths, half, G = (1, 40, 300), dim // 2 // 8 * 8, heads // kv
    c = eu.make_cache(lengths, kv, dim, 32, 5, evicts=True)
    g, (large_q, large_k) = seeded(6), LARGE[act]
    sign = torch.where(torch.rand((3, kv, 1, half), generator=g, device="cuda") < 0.5, -1.0, 1.0)
    q = torch.randn((3, kv, G, dim), generator=g, device="cuda")
    # mantissas just past halfway to the next of 8 bits: the first part is the next one and the rest negative
    rest = {"against": 0.625, "along": 0.375}.get(part)
    if rest is None:
        rest = torch.where(torch.rand((3, kv, G, half), generator=g, device="cuda") < 0.5, 0.625, 0.375)
    step = torch.randint(0, 64, (3, kv, G, half), generator=g, device="cuda") * 2.0
    q[..., :half] = sign * large_q * (1.0 + (step + rest) * 2.0 ** -7)
    far = []
    for b, n in enumerate(lengths):
        k = torch.randn((kv, n, dim), generator=g, device="cuda")
        k[:, :, :half] = 0.0
        t = torch.arange(n, device="cuda") % 3 == 1 if n > 1 else torch.zeros(n, dtype=torch.bool, device="cuda")
        k[:, t, :half] = -sign[b] * large_k * (1.0 + torch.rand((kv, int(t.sum()), half), generator=g, device="cuda"))
        eu.put(c, "k", b, k)
        far.append(t.cpu().numpy())
    q = q.reshape(3, heads * dim).to(DT[act])
    before = [eu.get(c, "weights", b, n) for b, n in enumerate(lengths)]
    out = torch.full_like(q, float("nan"))
    m.mosaic_cache_attend(c, q, heads, out, accumulate=True)
    got, qs, scale = f64(out).reshape(3, heads, dim), f64(q).reshape(3, heads, dim), dim ** -0.5
    for b, n in enumerate(lengths):
        near = ~far[b]
        k, v, now = eu.get(c, "k", b, n), eu.get(c, "v", b, n), eu.get(c, "weights", b, n)
        for h in range(kv):
            rows = qs[b, h * G: (h + 1) * G]
            assert (scale * (rows @ k[h][~near].T) < -2.0 ** 128).all()
            o, p = oc.attend(rows, k[h][near], v[h][near], scale)
            S = scale * (np.abs(rows) @ np.abs(k[h][near]).T).max(axis=1, keepdims=True)
            A = p @ np.abs(v[h][near])
            rel = (2 * (dim + 4) * S + n + 16) * U
            off = (rel + PARTS[act]) * A
            err = np.abs(got[b, h * G: (h + 1) * G] - o)
            assert (err <= off + UNIT[act] * (np.abs(o) + off) + TINY[act]).all(), (b, h, err.max())
            want = before[b][h][near] + p.sum(axis=0)
            assert (np.abs(now[h][near] - want) <= (rel * p).sum(axis=0) + 4 * U * want + 1e-38).all()
            assert np.array_equal(now[h][~near], before[b][h][~near])


def test_no_score_in_reach():
    """Every score -inf: zeros, and no weight."""
    for act in ("f32", "f16"):
        c = eu.make_cache((50,), 1, 64, 16, 7, evicts=True)
        large_q, large_k = LARGE[act]
        eu.put(c, "k", 0, torch.full((1, 50, 64), -large_k, device="cuda"))
        before = c.weights.clone()
        q = torch.full((1, 4 * 64), large_q * (1.0 + 0.625 * 2.0 ** -7), device="cuda").to(DT[act])
        out = torch.full_like(q, float("nan"))
        m.mosaic_cache_attend(c, q, 4, out, accumulate=True)
        assert not out.any()
        p, o = eu.where(c, 0, 0, 50)
        assert torch.equal(c.weights[p, :, o], before[p, :, o])
