"""Norm and rotation of queries and keys, the append to a paged cache and attention over it
(oracle, float64).

Test infrastructure.  The paper names the cache, its positions and grouped-query attention (Background,
omni model architecture) but no pages of several streams, head norms or frequency scaling; the
readings taken:
  * head norm: x_i w_i / sqrt(mean(x^2) + eps) over one head's values, before the rotation;
  * rotation of pair j by pos * theta_j, both halves scaled by a magnitude; pairings as in ``rope``;
  * token t of sequence s, the i-th of its m new ones, sits at row n - m + i of its n rows; row r is
    line r % P of page table[s][r // P];
  * attention of that token over the rows j <= n - m + i.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import chunk_attention
from .rope import pair_dims


def scaled_thetas(base, rot_dims, scaling="plain", factor=1.0, original_len=0.0, slow=1.0, fast=32.0):
    """Frequencies, one at a time."""
    out = []
    for j in range(rot_dims // 2):
        b = base
        if scaling == "base":
            b = base * factor ** (rot_dims / (rot_dims - 2))
        t = math.exp(-2.0 * j / rot_dims * math.log(b))
        if scaling == "linear":
            t = t / factor
        if scaling == "ramp":
            turns = original_len * t / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
            t = keep * t + (1.0 - keep) * t / factor
        out.append(t)
    return np.array(out)


def norm_rope(x, weight, eps, theta, pos, style, magnitude=1.0):
    """x [T, H, d] normed (weight [d] or None) and rotated (theta [R/2] or None) to pos [T]."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        mean = (x * x).sum(-1, keepdims=True) / x.shape[-1]
        x = x * np.asarray(weight, np.float64) / np.sqrt(mean + eps)
    if theta is None:
        return x
    a, b = pair_dims(2 * len(theta), style)
    phi = np.asarray(pos, np.float64)[:, None, None] * np.asarray(theta, np.float64)
    c, s = magnitude * np.cos(phi), magnitude * np.sin(phi)
    out = x.copy()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def gather_rows(pool, table_row, n):
    """Rows [0, n) of a sequence from pool [pages, P, H, d]."""
    page = pool.shape[1]
    return np.stack([pool[table_row[r // page], r % page] for r in range(n)]) if n else \
        np.zeros((0, *pool.shape[2:]), pool.dtype)


def ragged_attention(q, k_pool, v_pool, table, q_start, ctx_len, scale):
    """(out, spread) of q [T, H_q, d] float64 over float64 pools; spread[t, h, :] =
    sum_j p_j |v_j| + |out|, what an error of the probabilities is measured against.  Tokens of no
    sequence are NaN."""
    out = np.full(q.shape, np.nan)
    spread = np.full(q.shape, np.nan)
    for s, n in enumerate(ctx_len):
        t0, t1 = q_start[s], q_start[s + 1]
        if t1 == t0:
            continue
        k, v = gather_rows(k_pool, table[s], n), gather_rows(v_pool, table[s], n)
        out[t0:t1] = chunk_attention(q[t0:t1], k, v, scale)
        spread[t0:t1] = chunk_attention(q[t0:t1], k, np.abs(v), scale) + np.abs(out[t0:t1])
    return out, spread
