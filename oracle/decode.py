"""The decode step between the projections, in plain numpy and 64 bits: norm,
rotation and append, attention over a paged cache, and eviction.  Loops over
sequences and heads, written from the definitions; it shares no code with the
library."""
from __future__ import annotations

import math
from typing import Dict, Optional

import numpy as np

from . import formats as F


def transform(x, weight, eps, angles, interleaved):
    """A head [dim] in fp64: norm (with a weight), then rotation by `angles`, the
    rot / 2 cosines and sines of its position (or None).  Also returns the
    magnitude that rounding errors of the result are relative to."""
    y = np.asarray(x, np.float64).copy()
    if weight is not None:
        y = y / math.sqrt(np.mean(y * y) + eps) * np.asarray(weight, np.float64)
    size = np.abs(y)
    if angles is not None and len(angles):
        half = len(angles) // 2
        z = y.copy()
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = float(angles[i]), float(angles[half + i])
            z[a], z[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
            size[a], size[b] = abs(y[a] * c) + abs(y[b] * s), abs(y[b] * c) + abs(y[a] * s)
        y = z
    return y, size


def quantize_row(row32):
    """An fp32 row as e4m3 codes and a scale, by the per-token rule: IEEE fp32
    operations, nearest even.  A tiny row's codes are those of the row times a
    power of two, for which 448 / amax is a number."""
    x = np.asarray(row32, np.float32)
    a = np.max(np.abs(x))
    if a == 0:
        return np.zeros(x.shape, np.uint8), np.float32(0)
    up = np.float32(2.0 ** 60) if a < 2.0 ** -90 else np.float32(1)
    inv = np.float32(448) / (a * up)
    return F.e4m3_encode(x * up * inv), a / np.float32(448)


def attend(q, k, v, scale) -> Dict[str, np.ndarray]:
    """Heads of one key head: q [g, D], k and v [T, D].  Also the sizes that error
    bounds are relative to: sum |q k| of the largest score, and sum p |v|."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    g, D = q.shape
    if k.shape[0] == 0:
        z = np.zeros((g, D))
        return dict(out=z, lse=np.full(g, -np.inf), p=np.zeros((g, 0)), score_size=np.zeros(g), out_size=z)
    z = q @ k.T * scale
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    p = e / total
    return dict(out=p @ v, lse=(top + np.log(total))[:, 0], p=p,
                score_size=(np.abs(q) @ np.abs(k).T * abs(scale)).max(1), out_size=p @ np.abs(v))


def evict(weight, position, budget: int, recent: int, present=None):
    """One key head of one sequence: (kept slots that move, ascending; the freed
    slots they move to, ascending; weight and position afterwards).  Slots that
    are not present (their page is absent) are no places and are never kept:
    as many of the others stay as there are present slots below the budget."""
    n = len(weight)
    if n <= budget:
        return np.zeros(0, int), np.zeros(0, int), weight.copy(), position.copy()
    there = [t for t in range(n) if present is None or present[t]]
    newest = max([-1] + [int(position[t]) for t in there])
    slots = sorted(there, key=lambda t: (not position[t] > newest - recent, math.isnan(weight[t]),
                                         0.0 if math.isnan(weight[t]) else -float(weight[t]), t))
    places = [t for t in there if t < budget]
    kept = set(slots[:len(places)])
    to = np.array([t for t in places if t not in kept], int)
    of = np.array([t for t in there if t >= budget and t in kept], int)
    w, p = weight.copy(), position.copy()
    w[to], p[to] = weight[of], position[of]
    given_up = [t for t in there if t >= budget]
    w[given_up], p[given_up] = 0, -1
    return of, to, w, p


def gather(pool, table_row, n: int, head: int, page_size: int, scales: Optional[np.ndarray] = None):
    """The first n slots of a sequence from a [pages, heads, page_size, ...] pool, in fp64."""
    t = np.arange(n)
    page = np.asarray(table_row)[t // page_size]
    rows = np.asarray(pool, np.float64)[page, head, t % page_size]
    return rows if scales is None else rows * np.asarray(scales, np.float64)[page, head, t % page_size][:, None]
