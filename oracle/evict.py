"""Eviction by accumulated attention weight (oracle, float64 and exact integers).

Test infrastructure.  The paper's planner is metadata-only; this one ranks rows by the attention that
they were given.  The readings taken:
  * a row's weight is the sum, over the tokens that see it and all query heads, of their probabilities,
    added to `decay` times what it was;
  * above `high` rows exactly `budget` stay: the first `sink`, the last `recent`, and between them those of
    the largest weight, ties to the lower row, no-numbers last;
  * kept rows keep their order; row src[i] becomes row i.
"""
from __future__ import annotations

import math

import numpy as np


def row_weights(q, k, scale):
    """Weights [n] that the last m tokens' q [m, H_q, d] give to k [n, H_kv, d]."""
    m, hq, _ = q.shape
    n, hkv, _ = k.shape
    sees = np.arange(n)[None] <= np.arange(n - m, n)[:, None]
    total = np.zeros(n)
    for h in range(hq):
        x = np.where(sees, scale * (q[:, h] @ k[:, h // (hq // hkv)].T), -np.inf)
        p = np.exp(x - x.max(-1, keepdims=True))
        total += (p / p.sum(-1, keepdims=True)).sum(0)
    return total


def plan(weight, high, budget, sink, recent):
    """Rows kept of one sequence, in order."""
    n = len(weight)
    if n <= high:
        return list(range(n))
    rank = [-math.inf if math.isnan(w) else float(w) for w in weight]
    isnan = [math.isnan(w) for w in weight]
    middle = sorted(range(sink, n - recent), key=lambda r: (isnan[r], -rank[r], r))
    return (list(range(sink)) + sorted(middle[:budget - sink - recent]) + list(range(n - recent, n)))
