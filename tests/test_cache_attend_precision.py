"""In how many bits softmax weights meet the values (mosaic_cache_attend).

Over a 16-bit cache a weight is multiplied as a sum of 16-bit parts, each
rounded to nearest from what the ones before leave. A first part of p bits
leaves at most 2^-p of it, a second at most 2^-(2p + 1): 2^-17 of a weight for
two of bf16 (16-bit activations), 2^-23 for two of f16, nothing of 24 bits for
three of bf16 (float32 activations). Below f16's smallest step a part is off by
2^-25, in weights scaled so that the largest is at least 2^11: 2^-36 of the
weights' sum. So with A = sum p |v| an output is off by those times A (and
2^-36 sum |v| for f16), by the float32 terms of test_gpu_cache_attend.py, and by
its own rounding, which is all that 16 bits of activations show.

Values come in pairs of opposite sign with almost equal weights, so an output
is far smaller than A, and a lost part shows."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import mosaic as m
from tests.cache_util import DT, TINY, TYPES, UNIT, f64, get, make_cache, put, seeded

U = 2.0 ** -24
PARTS = {("bf16", "bf16"): (2, 2.0 ** -17, 0.0), ("f32", "bf16"): (3, 0.0, 0.0), ("f16", "f16"): (2, 2.0 ** -23, 2.0 ** -36),
         ("f32", "f16"): (2, 2.0 ** -23, 2.0 ** -36), ("f32", "f32"): (1, 0.0, 0.0)}


def tolerance(act, cache, q, k, v, scale, o, p):
    D, n = k.shape[1], len(k)
    _, unit, floor = PARTS[act, cache]
    S = abs(scale) * (np.abs(q) @ np.abs(k).T).max(axis=1, keepdims=True)
    A = p @ np.abs(v)
    off = ((2 * (D + 4) * S + n + 16) * U + unit) * A + floor * np.abs(v).sum(axis=0)
    return off + UNIT[act] * (np.abs(o) + off) + TINY[act]


def inputs(g, cache, kv, n, dim, device="cpu"):
    """Keys and values of n tokens in pairs."""
    k = torch.randn((kv, n, dim), generator=g, device=device)
    v = (torch.rand((kv, n, dim), generator=g, device=device) + 1.0).to(DT[cache])
    half = n // 2
    k[:, 1: 2 * half: 2] = k[:, 0: 2 * half: 2] + 0.02 * k[:, 1: 2 * half: 2]
    v[:, 1: 2 * half: 2] = -v[:, 0: 2 * half: 2]
    return k.to(DT[cache]), v


def emulated(act, cache, q, k, v, scale, parts):
    """The kernel's arithmetic in float64 but for the weights' parts."""
    s = scale * (q @ k.T) / np.log(2.0)
    w = np.exp2(s - s.max(axis=1, keepdims=True)) * (2.0 ** 11 if cache == "f16" else 1.0)
    rest, total = torch.from_numpy(w).clone(), torch.zeros_like(torch.from_numpy(w))
    for _ in range(parts):
        part = rest.float().to(DT[cache]).double()
        total += part
        rest -= part
    o = (total.numpy() @ v) / w.sum(axis=1, keepdims=True)
    return torch.from_numpy(o).float().to(DT[act]).double().numpy()


@pytest.mark.parametrize("act,cache", [t for t in PARTS if t[1] != "f32"])
def test_the_bound_tells_the_parts_apart(act, cache):
    """On the host: it holds for as many parts as there should be, and not for
    one part fewer."""
    parts = PARTS[act, cache][0]
    bad = 0
    for seed in range(12):
        g = torch.Generator().manual_seed(seed)
        n, dim = (2, 4, 6)[seed % 3], 8
        k, v = (t[0].double().numpy() for t in inputs(g, cache, 1, n, dim))
        q = (0.3 * torch.randn((16, dim), generator=g)).to(DT[act]).double().numpy()
        o, p = oc.attend(q, k, v, 0.1)
        tol = tolerance(act, cache, q, k, v, 0.1, o, p)
        assert (np.abs(emulated(act, cache, q, k, v, 0.1, parts) - o) <= tol).all()
        bad += (np.abs(emulated(act, cache, q, k, v, 0.1, parts - 1) - o) > tol).sum()
    assert bad > 0


@pytest.mark.gpu
@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("heads,kv,dim", ((16, 2, 8), (4, 2, 64), (8, 1, 128), (40, 1, 80), (3, 3, 256)))
@pytest.mark.parametrize("std,scale", ((0.3, 0.1), (1.0, 0.3)))
def test_weights_are_not_rounded_to_16_bits(act, cache, heads, kv, dim, std, scale):
    lengths = (2, 4, 17, 40, 130)
    c = make_cache(lengths, kv, dim, 16, cache, 5)
    g = seeded(6)
    for b, n in enumerate(lengths):
        for name, x in zip("kv", inputs(g, cache, kv, n, dim, "cuda")):
            put(c, name, b, x)
    q = (std * torch.randn((len(lengths), heads * dim), generator=g, device="cuda")).to(DT[act])
    out = torch.full_like(q, float("nan"))
    m.mosaic_cache_attend(c, q, heads, out, scale=scale)
    got, qs, G = f64(out).reshape(-1, heads, dim), f64(q).reshape(-1, heads, dim), heads // kv
    for b, n in enumerate(lengths):
        k, v = get(c, "k", b, n), get(c, "v", b, n)
        for h in range(kv):
            rows = qs[b, h * G: (h + 1) * G]
            o, p = oc.attend(rows, k[h], v[h], scale)
            tol = tolerance(act, cache, rows, k[h], v[h], scale, o, p)
            err = np.abs(got[b, h * G: (h + 1) * G] - o)
            assert (err <= tol).all(), (b, h, (err / tol).max())
