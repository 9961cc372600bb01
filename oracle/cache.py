"""Cached decoding on the trusted client in float64 (numpy), from the
definitions of include/mosaic_cache.h: rotary positions, attention of one
token, eviction by accumulated weight. One sequence, and for the last two one
key/value head, at a time; pages are none of its business."""
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
