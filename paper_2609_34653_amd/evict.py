"""Thin Python binding of the calls that evict by attention weight, of libomnitide.so
(include/omnitide_evict.h).

As in ``paged``: each function has the name of the C entry point it calls, checks its tensors, passes
the current HIP stream, and raises ``OmnitideError`` with the library's status code on failure; every
step of the computation runs in the HIP kernels.

Shapes: pools bf16 [n_pages, page_size, H_kv, d], or [n_pages, page_size, R + 64] of a latent cache (one
KV head); weights float32 [n_seq, rows], whose rows may be strided; page_table, q_start and ctx_len as
in ``paged``.
"""
from __future__ import annotations

import ctypes

import torch

from . import omnitide as ot
from . import paged as pg
from .latent import _mat, _pool
from .omnitide import ROPE_HALF, ROPE_INTERLEAVED, OmnitideError, _check  # noqa: F401
from .paged import _dev, _device, _on, _status, _table, _theta, _ws

EXPORTS = ("omnitide_paged_attn_weights", "omnitide_paged_attn_weights_workspace_bytes",
           "omnitide_evict_plan", "omnitide_evict_plan_workspace_bytes", "omnitide_paged_compact")

_P, _I, _SZ, _L, _F = pg._P, pg._I, pg._SZ, pg._L, pg._F
_T, _BF16, _F32, _I32 = pg._T, pg._BF16, pg._F32, pg._I32

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded HIP library with the eviction calls declared."""
    global _lib
    if _lib is None:
        L = ot.lib()
        L.omnitide_paged_attn_weights.argtypes = [_P, _P, _I, _I, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _F,
                                                  _F, _P, _P, _P, _L, _P, _SZ, _P, _P]
        L.omnitide_paged_attn_weights_workspace_bytes.argtypes = [_I] * 7
        L.omnitide_evict_plan.argtypes = [_P, _L, _P, _I, _I, _I, _I, _I, _I, _P, _L, _P, _P, _L, _P, _SZ, _P,
                                          _P]
        L.omnitide_evict_plan_workspace_bytes.argtypes = [_I, _I]
        L.omnitide_paged_compact.argtypes = [_P, _P, _I, _I, _I, _I, _P, _I, _P, _P, _I, _P, _L, _P, _I, _P, _I,
                                             _I, _I, _P, _P]
        for name in ("omnitide_paged_attn_weights_workspace_bytes",
                     "omnitide_evict_plan_workspace_bytes"):
            getattr(L, name).restype = _SZ
        for name in ("omnitide_paged_attn_weights", "omnitide_evict_plan", "omnitide_paged_compact"):
            getattr(L, name).restype = _I
        _lib = L
    return _lib


def _kv_heads(pool):
    """(H_kv, d) of a pool's rows."""
    if pool.dim() == 3:
        return 1, pool.shape[2]
    if pool.dim() != 4:
        raise ValueError("a pool must be [n_pages, page_size, H_kv, d] or [n_pages, page_size, d]")
    return pool.shape[2], pool.shape[3]


def omnitide_paged_attn_weights_workspace_bytes(n_tokens, n_seq, max_ctx, max_q, n_q_heads, n_kv_heads,
                                                head_dim) -> int:
    return int(lib().omnitide_paged_attn_weights_workspace_bytes(n_tokens, n_seq, max_ctx, max_q,
                                                                 n_q_heads, n_kv_heads, head_dim))


def omnitide_paged_attn_weights(q, k_pool, page_table, q_start, ctx_len, max_q, scale, weight_out,
                                weight_in=None, seen_len=None, decay=1.0, workspace=None, d_status=None,
                                stream=None):
    """The weight that q [tokens, H_q, d] bf16 gives to each row, over heads and tokens, added to
    decay * weight_in; weight_out [n_seq, rows] float32 (may be weight_in)."""
    dev = _device(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, H_q, d]")
    n, hq, d = q.shape
    at, n_pages, page, _ = _pool(k_pool, "k_pool", dev)
    hkv, dp = _kv_heads(k_pool)
    if dp != d:
        raise ValueError("the pool does not match q")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    wo = _mat(weight_out, "weight_out", _F32, dev)
    if wo[1] != n_seq or wo[2] < max_pages * page:
        raise ValueError("weight_out must have a row per sequence, of max_pages * page_size at least")
    wi = None
    if weight_in is not None:
        m = _mat(weight_in, "weight_in", _F32, dev)
        if m[1:] != wo[1:]:
            raise ValueError("weight_in must have weight_out's shape and strides")
        wi = m[0]
    _check((_lib or lib()).omnitide_paged_attn_weights(
        _dev(q, "q", _BF16, q.numel(), dev), at, n_pages, page, tab, max_pages,
        _dev(q_start, "q_start", _I32, n_seq + 1, dev), ctx, n_seq, n, int(max_q), hq, hkv, d, scale, decay,
        None if seen_len is None else _dev(seen_len, "seen_len", _I32, n_seq, dev), wi, wo[0], wo[3],
        *_ws(workspace, dev), _status(d_status, dev), _on(q, stream)), "omnitide_paged_attn_weights")


def omnitide_evict_plan_workspace_bytes(n_seq, max_ctx) -> int:
    return int(lib().omnitide_evict_plan_workspace_bytes(n_seq, max_ctx))


def omnitide_evict_plan(weight, ctx_len, high, budget, sink, recent, src_row, new_len, weight_out=None,
                        workspace=None, d_status=None, stream=None):
    """The rows kept of each sequence: src_row [n_seq, >= high] int32, new_len [n_seq] int32 and, if
    given, their weights in weight_out [n_seq, >= high]."""
    dev = _device(weight, "weight")
    w, src = _mat(weight, "weight", _F32, dev), _mat(src_row, "src_row", _I32, dev)
    n_seq = w[1]
    wo = (None, n_seq, 0, 0) if weight_out is None else _mat(weight_out, "weight_out", _F32, dev)
    if src[1] != n_seq or wo[1] != n_seq:
        raise ValueError("weight, src_row and weight_out must have a row per sequence")
    if src[2] < high or (wo[0] is not None and wo[2] < high):
        raise ValueError("src_row and weight_out must hold `high` rows per sequence")
    _check((_lib or lib()).omnitide_evict_plan(
        w[0], w[3], _dev(ctx_len, "ctx_len", _I32, n_seq, dev), n_seq, w[2], int(high), int(budget),
        int(sink), int(recent), src[0], src[3], _dev(new_len, "new_len", _I32, n_seq, dev), wo[0], wo[3],
        *_ws(workspace, dev), _status(d_status, dev), _on(weight, stream)), "omnitide_evict_plan")


def omnitide_paged_compact(k_pool, v_pool, page_table, ctx_len, dst_table, src_row, new_len, theta=None,
                           rope_style=ROPE_HALF, rope_offset=0, d_status=None, stream=None):
    """Row src_row[s, i] of each sequence becomes its row i in the pages of dst_table (all in the same
    pools; v_pool None: keys alone), its key turned to its new place if theta is given."""
    dev = _device(k_pool, "k_pool")
    at, n_pages, page, row = _pool(k_pool, "k_pool", dev)
    hkv, d = _kv_heads(k_pool)
    if v_pool is not None and (not isinstance(v_pool, _T) or v_pool.shape != k_pool.shape):
        raise ValueError("v_pool must have k_pool's shape")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    if not (isinstance(dst_table, _T) and dst_table.dim() == 2 and dst_table.shape[0] == n_seq):
        raise ValueError("dst_table must be [n_seq, max_pages]")
    src = _mat(src_row, "src_row", _I32, dev)
    if src[1] != n_seq:
        raise ValueError("src_row must have a row per sequence")
    # (of a strided src_row, rows beyond its width are not the caller's)
    if src[3] != src[2] and n_seq > 1:
        raise ValueError("src_row must be contiguous")
    th, dims = _theta(theta)
    _check((_lib or lib()).omnitide_paged_compact(
        at, None if v_pool is None else _dev(v_pool, "v_pool", _BF16, v_pool.numel(), dev), n_pages, page,
        hkv, d, tab, max_pages, ctx, _dev(dst_table, "dst_table", _I32, dst_table.numel(), dev),
        dst_table.shape[1], src[0], src[3], _dev(new_len, "new_len", _I32, n_seq, dev), n_seq, th, dims,
        rope_style, int(rope_offset), _status(d_status, dev), _on(k_pool, stream)),
        "omnitide_paged_compact")
