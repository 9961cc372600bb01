"""Cached decoding on the trusted client in float64 (numpy), from the
definitions of include/mosaic_cache.h: rotary positions, norms, rows in 4 bits,
attention of one token, eviction by accumulated weight. One sequence, and for
attention and eviction one key/value head, at a time; pages are none of its
business."""
from __future__ import annotations

import numpy as np


def rotate(x, table, places, sections, interleaved):
    """x (tokens x heads x dim) with the pairs of axis a turned by the row
    places[a, t] of the table (the nearest row for a place outside it)."""
    y = np.array(x, dtype=np.float64)
    P = sum(sections)
    j = 0
    for axis, count in enumerate(sections):
        row = np.clip(np.asarray(places[axis], dtype=np.int64), 0, len(table) - 1)
        for _ in range(count):
            lo, hi = (2 * j, 2 * j + 1) if interleaved else (j, P + j)
            c, s = table[row, j].astype(np.float64)[:, None], table[row, P + j].astype(np.float64)[:, None]
            y[:, :, lo] = x[:, :, lo] * c - x[:, :, hi] * s
            y[:, :, hi] = x[:, :, hi] * c + x[:, :, lo] * s
            j += 1
    return y


def attend(q, k, v, scale):
    """q (group x dim), k and v (tokens x dim): the outputs (group x dim) and
    the attention weights (group x tokens); zeros without tokens of a score
    above -inf."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros((len(q), v.shape[1])), np.zeros((len(q), 0))
    s = scale * (q @ k.T)
    top = s.max(axis=1, keepdims=True)
    p = np.exp(s - np.where(top == -np.inf, 0.0, top))
    total = p.sum(axis=1, keepdims=True)
    p /= np.where(total == 0.0, 1.0, total)
    return p @ v, p


def evict(weights, order, seen, budget, recent, there=None):
    """The slot that the token of each slot had before: weights and order by
    slot, of all the tokens held. ``there``: which slots have a page (None:
    all); -1 for one that does not."""
    n = len(weights)
    there = [True] * n if there is None else list(there)
    if n <= budget:
        return [i if there[i] else -1 for i in range(n)]
    def rank(i):
        w = float(weights[i])
        if order[i] >= seen - recent:
            return (0, 0.0, i)
        return (2, 0.0, i) if np.isnan(w) else (1, -w, i)
    room = [i for i in range(budget) if there[i]]
    stay = sorted(sorted((i for i in range(n) if there[i]), key=rank)[:len(room)])
    inside = {i for i in stay if i < budget}
    movers = iter(i for i in stay if i >= budget)
    return [-1 if not there[i] else i if i in inside else next(movers) for i in range(budget)]


def normalise(x, weight, eps):
    """x (... x dim) over its root mean square, times weight."""
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)


E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(dim):
    return -(-(dim // 2 + dim // 8) // 16) * 16


def to_e2m1(x):
    """Codes (... x dim) and scales (... x dim / 8) of x: the least power of two
    from 2^-126 to 2^125 under which no magnitude of 8 is over 7, the nearest
    codes with the sign of x (of a zero too), an even one between two; scale 255
    where one is not finite."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 8, 8)
    top = np.abs(g).max(axis=-1)
    scale = np.full(top.shape, 255, dtype=np.int64)
    fine = np.isfinite(top)
    e = np.full(int(fine.sum()), 252)
    for byte in range(251, 0, -1):
        e = np.where(top[fine] <= 7.0 * 2.0 ** (byte - 127), byte, e)
    scale[fine] = e
    a = np.where(fine[..., None], np.abs(g), 0.0) * 2.0 ** (127.0 - np.where(fine, scale, 127))[..., None]
    far = np.abs(a[..., None] - E2M1)
    best = far.min(axis=-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])          # even codes first
    code = order[np.argmax(far[..., order] == best, axis=-1)] + 8 * np.signbit(g)
    return np.where(fine[..., None], code, 0).reshape(x.shape), scale


def pack_e2m1(codes, scales):
    dim = codes.shape[-1]
    out = np.zeros((*codes.shape[:-1], row_bytes(dim)), dtype=np.uint8)
    out[..., : dim // 2] = codes[..., 0::2] + 16 * codes[..., 1::2]
    out[..., dim // 2: dim // 2 + dim // 8] = scales
    return out


def unpack_e2m1(rows, dim):
    """The values that rows of bytes stand for."""
    rows = np.asarray(rows).astype(np.int64)
    codes = np.stack([rows[..., : dim // 2] % 16, rows[..., : dim // 2] // 16], axis=-1).reshape(*rows.shape[:-1], dim)
    scale = rows[..., dim // 2: dim // 2 + dim // 8]
    value = E2M1[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    factor = np.where(scale == 255, np.nan, 2.0 ** (np.where(scale == 255, 127, scale) - 127.0))
    return (value.reshape(*rows.shape[:-1], dim // 8, 8) * factor[..., None]).reshape(*rows.shape[:-1], dim)
