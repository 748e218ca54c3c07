"""CPU oracle for the calls over caches in pages.  TEST INFRASTRUCTURE ONLY.

Plain float64 statements of what a slot holds and what the calls compute, one (sequence, kv-head) or one row at a time;
they share no code with the HIP path.  Readings:
  R19 Generation over a compressed cache (Section 4.4 times it, the paper does not restate it): a new token's key and
      value join the cache of every head, attention runs over all slots, order does not matter to it.
  R20 Eviction by accumulated attention weight, the baseline family the paper compares with (H2O): per kv-head, the
      weight of a token is the plain sum of its softmax weights over steps and over the query heads of the kv-head, the
      newest positions are kept in any case, ties go to the lower slot; kept slots move only out of the part that is cut off.
"""
from __future__ import annotations

import math

import numpy as np


def norm_and_rotate(x, weight, eps, position, inv_freq, interleaved):
    """One head's row in float64: root-mean-square norm with a weight (None: none), then rotation of the first 2 len(inv_freq) elements."""
    y = np.asarray(x, dtype=np.float64).copy()
    if weight is not None:
        y = y / math.sqrt(float(np.mean(y * y)) + eps) * np.asarray(weight, dtype=np.float64)
    if inv_freq is None:
        return y
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = math.fmod(float(position) * float(inv_freq[i]), 2 * math.pi)
        c, s = math.cos(angle), math.sin(angle)
        y[a], y[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
    return y


def slot_row(pool, table_row, n_pages, page_tokens, h, slot):
    """Row of a slot in a [pages][heads][page_tokens][d] pool; None where its page is not there."""
    page = int(table_row[slot // page_tokens])
    return pool[page, h, slot % page_tokens] if 0 <= page < n_pages else None


def attention(q, k, v, scale):
    """q [g][d]; k, v [n][d], the rows that are there.  -> out [g][d], lse [g], weights [g][n]."""
    g, n = len(q), len(k)
    if n == 0:
        return np.zeros((g, q.shape[1])), np.full(g, -np.inf), np.zeros((g, 0))
    x = scale * np.asarray(q, dtype=np.float64) @ np.asarray(k, dtype=np.float64).T
    top = x.max(axis=1, keepdims=True)
    e = np.exp(x - top)
    p = e / e.sum(axis=1, keepdims=True)
    return p @ np.asarray(v, dtype=np.float64), top[:, 0] + np.log(e.sum(axis=1)), p


def evict(weight, pos, n, budget, recent):
    """-> (new number of slots, [(from, to)] moves) of one head; weight and pos are its slots' arrays."""
    if n <= budget:
        return n, []
    newest = max(int(pos[s]) for s in range(n))
    order = sorted(range(n), key=lambda s: (0 if int(pos[s]) > newest - recent else 1, 0.0 if int(pos[s]) > newest - recent else -float(weight[s]), s))
    kept = sorted(order[:budget])
    stay = {s for s in kept if s < budget}
    return budget, list(zip([s for s in kept if s >= budget], [s for s in range(budget) if s not in stay]))
