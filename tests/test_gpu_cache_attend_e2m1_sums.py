"""Weights added up over a cache in 4 bits are p = exp(s) / sum exp(s) with a sum of
float32 weights, whatever the parts leave out that multiply the values: to (2 (dim +
4) S + n + 16) 2^-24 p each, as in test_gpu_cache_attend.py, for activations of 16
bits too."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests import e2m1_util as eu
from tests.cache_util import f64
from tests.test_gpu_cache_attend_e2m1 import U, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("heads,kv,dim", ((64, 64, 8), (96, 32, 16), (64, 8, 64), (30, 2, 80), (40, 2, 128)))
def test_weights_of_few_tokens(act, heads, kv, dim):
    lengths, G = (2, 3, 4, 5, 7, 11), heads // kv
    c = eu.make_cache(lengths, kv, dim, 16, 5, evicts=True, scale=0.1)
    c.weights.zero_()
    q, _, scale = run(c, heads, act, 6, accumulate=True, std=0.5)
    qs = f64(q).reshape(-1, heads, dim)
    for b, n in enumerate(lengths):
        k, v, now = eu.get(c, "k", b, n), eu.get(c, "v", b, n), eu.get(c, "weights", b, n)
        for h in range(kv):
            rows = qs[b, h * G: (h + 1) * G]
            p = oc.attend(rows, k[h], v[h], scale)[1]
            S = scale * (np.abs(rows) @ np.abs(k[h]).T).max(axis=1, keepdims=True)
            rel = (2 * (dim + 4) * S + n + 16) * U
            off = np.abs(now[h] - p.sum(axis=0))
            assert (off <= (rel * p).sum(axis=0) + 4 * U * p.sum(axis=0)).all(), (b, h, (off / p.sum(axis=0)).max())
