"""A latent cache and its attention in both forms (oracle, float64).

Test infrastructure.  The paper's cache holds keys and values per head; a latent cache holds one row for all
heads.  The readings taken:
  * row: the latent, normed as a whole (x_i w_i / sqrt(mean(x^2) + eps)), then the key part, rotated;
  * absorbed: every head's query meets the whole row, and the value is the row's latent;
  * expanded: head h has keys and values of its own, a key's score is that of the head's part plus that
    of the rotated part, which all heads share;
  * a sequence's tokens are its last rows, and token t sees the rows up to its own.
"""
from __future__ import annotations

import numpy as np

from .paged import gather_rows, norm_rope


def latent_row(latent, k_rope, weight, eps, theta, pos, style, magnitude=1.0):
    """Rows [T, R + E] of latents [T, R] and key parts [T, E]."""
    x = norm_rope(np.asarray(latent, np.float64)[:, None], weight, eps, None, pos, style)[:, 0]
    e = norm_rope(np.asarray(k_rope, np.float64)[:, None], None, 0.0, theta, pos, style, magnitude)[:, 0]
    return np.concatenate([x, e], -1)


def _softmax(x):
    x = np.exp(x - x.max(-1, keepdims=True))
    return x / x.sum(-1, keepdims=True)


def absorbed_attention(q, rows, latent_dim, scale):
    """(out, spread) [m, H, R] of the last m tokens' q [m, H, R + E] over rows [n, R + E]; spread =
    sum_j p_j |c_j| + |out|."""
    m, n = q.shape[0], rows.shape[0]
    out, spread = (np.zeros((m, q.shape[1], latent_dim)) for _ in range(2))
    for i in range(m):
        seen = rows[:n - m + i + 1]
        p = _softmax(scale * (q[i] @ seen.T))
        out[i] = p @ seen[:, :latent_dim]
        spread[i] = p @ np.abs(seen[:, :latent_dim]) + np.abs(out[i])
    return out, spread


def expanded_attention(q, k, v, k_rope, scale):
    """(out, spread) [m, H, d] of the last m tokens' q [m, H, d + E] over k, v [n, H, d] and k_rope [n, E]."""
    m, n, d = q.shape[0], k.shape[0], k.shape[2]
    out, spread = (np.zeros((m, q.shape[1], d)) for _ in range(2))
    sees = np.arange(n)[None] <= np.arange(n - m, n)[:, None]
    for h in range(q.shape[1]):
        x = scale * (q[:, h, :d] @ k[:, h].T + q[:, h, d:] @ k_rope.T)
        p = _softmax(np.where(sees, x, -np.inf))
        out[:, h] = p @ v[:, h]
        spread[:, h] = p @ np.abs(v[:, h]) + np.abs(out[:, h])
    return out, spread


__all__ = ["latent_row", "absorbed_attention", "expanded_attention", "gather_rows"]
