"""Thin Python binding of the latent-cache calls of libomnitide.so (include/omnitide_latent.h).

As in ``paged``: each function has the name of the C entry point it calls, checks its tensors, passes
the current HIP stream, and raises ``OmnitideError`` with the library's status code on failure; every
step of the computation runs in the HIP kernels.

Shapes: pool bf16 [n_pages, page_size, R + 64], a latent of R values and a key part of 64 per row;
page_table, q_start and ctx_len as in ``paged``.  Where a call takes strides, parts of one projection's
output (views whose last dimension is contiguous) can be passed.
"""
from __future__ import annotations

import ctypes

import torch

from . import omnitide as ot
from . import paged as pg
from .omnitide import BF16, F32, ROPE_HALF, ROPE_INTERLEAVED, OmnitideError, _check, _kv_dtype  # noqa: F401
from .paged import _dev, _device, _float_type, _on, _out, _same, _status, _table, _theta, _ws

ROPE_DIM = 64

EXPORTS = ("omnitide_latent_append", "omnitide_paged_rows", "omnitide_latent_decode_attn",
           "omnitide_latent_decode_workspace_bytes", "omnitide_latent_chunk_attn",
           "omnitide_latent_chunk_attn_workspace_bytes")

_P, _I, _SZ, _L, _F = pg._P, pg._I, pg._SZ, pg._L, pg._F
_T, _BF16, _I32 = pg._T, pg._BF16, pg._I32

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded HIP library with the latent calls declared."""
    global _lib
    if _lib is None:
        L = ot.lib()
        L.omnitide_latent_append.argtypes = [_P, _P, _P, _I, _I, _I, _I, _L, _L, _L, _L, _P, _I, _I, _P,
                                             _I, _P, _P, _I, _P, _P, _F, _P, _I, _F, _P, _L, _L, _P, _P]
        L.omnitide_paged_rows.argtypes = [_P, _I, _I, _I, _P, _I, _P, _P, _I, _I, _P, _L, _P, _P]
        L.omnitide_latent_decode_attn.argtypes = [_P, _P, _I, _I, _P, _I, _P, _I, _I, _I, _I, _F, _P, _I,
                                                  _P, _SZ, _P, _P]
        L.omnitide_latent_chunk_attn.argtypes = [_P, _P, _P, _P, _L, _L, _L, _L, _L, _P, _P, _I, _I, _I, _I,
                                                 _I, _F, _P, _I, _P, _SZ, _P, _P]
        for name in ("omnitide_latent_decode_workspace_bytes",
                     "omnitide_latent_chunk_attn_workspace_bytes"):
            getattr(L, name).argtypes = [_I] * 5
            getattr(L, name).restype = _SZ
        for name in ("omnitide_latent_append", "omnitide_paged_rows", "omnitide_latent_decode_attn",
                     "omnitide_latent_chunk_attn"):
            getattr(L, name).restype = _I
        _lib = L
    return _lib


# ----------------------------------------------------------------------------- marshalling

def _strided(t, name: str, dtype, dev: int, dims: int):
    """Address of a tensor of `dims` dimensions of dtype whose last one is contiguous."""
    if not (type(t) is _T and t.dtype is dtype and t.get_device() == dev and t.dim() == dims):
        if not isinstance(t, _T):
            raise TypeError(f"{name} must be a tensor")
        if t.dtype is not dtype:
            raise TypeError(f"{name}: dtype {t.dtype} is not {dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        _same(t, name, dev)
        if t.dim() != dims:
            raise ValueError(f"{name} must have {dims} dimensions")
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr()


def _mat(t, name: str, dtype, dev: int):
    """(address, rows, width, row stride) of a matrix with contiguous rows."""
    if type(t) is _T and t.dtype is dtype and t.get_device() == dev:
        shape, stride = t.shape, t.stride()
        if len(shape) == 2 and stride[1] == 1:
            return t.data_ptr(), shape[0], shape[1], stride[0] if shape[0] > 1 else shape[1]
    at = _strided(t, name, dtype, dev, 2)
    n, w = t.shape
    return at, n, w, t.stride(0) if n > 1 else w


def _heads(t, name: str, dtype, dev: int):
    """(address, rows, heads, width, row stride, head stride) of [rows, heads, width]."""
    if type(t) is _T and t.dtype is dtype and t.get_device() == dev:
        shape, stride = t.shape, t.stride()
        if len(shape) == 3 and stride[2] == 1 and shape[0] > 1 and shape[1] > 1:
            return t.data_ptr(), *shape, stride[0], stride[1]
    at = _strided(t, name, dtype, dev, 3)
    n, h, w = t.shape
    hs = t.stride(1) if h > 1 else w
    return at, n, h, w, t.stride(0) if n > 1 else max((h - 1) * hs + w, 0), hs


def _pool(pool, name: str, dev: int):
    """(address, n_pages, page_size, row elements) of a pool [n_pages, page_size, ...]."""
    if type(pool) is _T and pool.dtype is _BF16 and pool.get_device() == dev and pool.is_contiguous():
        shape = pool.shape
        if len(shape) == 3:
            return pool.data_ptr(), *shape
        if len(shape) == 4:
            return pool.data_ptr(), shape[0], shape[1], shape[2] * shape[3]
    if not (isinstance(pool, _T) and pool.dim() >= 3):
        raise ValueError(f"{name} must be [n_pages, page_size, ...]")
    at = _dev(pool, name, _BF16, pool.numel(), dev)
    n_pages, page = pool.shape[:2]
    row = pool.shape[2]
    for x in pool.shape[3:]:
        row *= x
    return at, n_pages, page, row


# ----------------------------------------------------------------------------------- calls

def omnitide_latent_append(latent, k_rope, pool, page_table, q_start, ctx_len, pos=None, theta=None,
                           rope_style=ROPE_HALF, magnitude=1.0, latent_weight=None, eps=1e-6, q_rope=None,
                           q_out=None, d_status=None, stream=None):
    """The new tokens' latent [tokens, R] (normed) and k_rope [tokens, 64] (rotated) into the pages;
    q_rope [tokens, heads, 64] rotated into q_out (bf16) if given."""
    dt = _float_type(latent, "latent")
    dev = _device(latent, "latent")
    li, ki = _mat(latent, "latent", dt, dev), _mat(k_rope, "k_rope", dt, dev)
    n, R = li[1:3]
    if ki[1:3] != (n, ROPE_DIM):
        raise ValueError(f"k_rope must be [{n}, {ROPE_DIM}]")
    qi = qo = (None, 0, 0, 0, 0, 0)
    if q_rope is not None or q_out is not None:
        qi, qo = _heads(q_rope, "q_rope", dt, dev), _heads(q_out, "q_out", _BF16, dev)
        if qi[1] != n or qi[3] != ROPE_DIM or qi[1:4] != qo[1:4]:
            raise ValueError("q_rope, q_out and latent do not match")
    at, n_pages, page, row = _pool(pool, "pool", dev)
    if row != R + ROPE_DIM:
        raise ValueError("the pool does not match latent")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    th, dims = _theta(theta)
    if theta is not None and dims != ROPE_DIM:
        raise ValueError(f"theta must hold {ROPE_DIM // 2} frequencies")
    _check((_lib or lib()).omnitide_latent_append(
        li[0], ki[0], qi[0], BF16 if dt is _BF16 else F32, n, qi[2], R, li[3], ki[3], qi[4], qi[5], at,
        n_pages, page, tab, max_pages, _dev(q_start, "q_start", _I32, n_seq + 1, dev), ctx, n_seq,
        None if pos is None else _dev(pos, "pos", _I32, n, dev),
        None if latent_weight is None else _dev(latent_weight, "latent_weight", dt, R, dev), eps, th,
        rope_style, magnitude, qo[0], qo[4], qo[5], _status(d_status, dev), _on(latent, stream)),
        "omnitide_latent_append")


def omnitide_paged_rows(pool, page_table, row_start, ctx_len, out, d_status=None, stream=None):
    """Rows [0, row_start[s + 1] - row_start[s]) of each sequence from pool [n_pages, page_size, ...]
    into out [rows, row elements] (rows may be strided)."""
    dev = _device(out, "out")
    at, n_pages, page, row = _pool(pool, "pool", dev)
    o = _mat(out, "out", _BF16, dev)
    if o[2] != row:
        raise ValueError("out does not match the pool's rows")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    _check((_lib or lib()).omnitide_paged_rows(
        at, n_pages, page, row, tab, max_pages, _dev(row_start, "row_start", _I32, n_seq + 1, dev), ctx,
        n_seq, o[1], o[0], o[3], _status(d_status, dev), _on(out, stream)), "omnitide_paged_rows")


def omnitide_latent_decode_workspace_bytes(n_seq, n_q, max_ctx, n_heads, latent_dim) -> int:
    return int(lib().omnitide_latent_decode_workspace_bytes(n_seq, n_q, max_ctx, n_heads, latent_dim))


def omnitide_latent_decode_attn(q, pool, page_table, ctx_len, scale, out, workspace=None, d_status=None,
                                stream=None):
    """q [n_seq, n_q, heads, R + 64] bf16 (absorbed) of the last n_q tokens of each sequence; out
    [n_seq, n_q, heads, R] float32 or bf16.  A sequence with ctx_len 0 is idle: zeros."""
    dev = _device(q, "q")
    if q.dim() != 4:
        raise ValueError("q must be [n_seq, n_q, heads, R + 64]")
    n_seq, nq, h, w = q.shape
    at, n_pages, page, row = _pool(pool, "pool", dev)
    tab, max_pages, ctx, ns = _table(page_table, ctx_len, dev)
    if row != w or ns != n_seq:
        raise ValueError("the pool or the table does not match q")
    R = w - ROPE_DIM
    args = (_dev(q, "q", _BF16, q.numel(), dev), at, n_pages, page, tab, max_pages, ctx, n_seq, nq, h, R,
            scale, _out(out, n_seq * nq * h * R, dev), _kv_dtype(out), *_ws(workspace, dev),
            _status(d_status, dev))
    _check((_lib or lib()).omnitide_latent_decode_attn(*args, _on(q, stream)),
           "omnitide_latent_decode_attn")


def omnitide_latent_chunk_attn_workspace_bytes(n_tokens, n_seq, n_rows, n_heads, head_dim) -> int:
    return int(lib().omnitide_latent_chunk_attn_workspace_bytes(n_tokens, n_seq, n_rows, n_heads,
                                                                head_dim))


def omnitide_latent_chunk_attn(q, k, v, k_rope, q_start, kv_start, scale, out, workspace=None,
                               d_status=None, stream=None):
    """q [tokens, heads, d + 64] bf16 over expanded k and v [rows, heads, d] and the shared k_rope
    [rows, 64] of a ragged batch of chunks; out [tokens, heads, d] float32 or bf16."""
    dev = _device(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, d + 64]")
    n, h, w = q.shape
    ki, vi = _heads(k, "k", _BF16, dev), _heads(v, "v", _BF16, dev)
    ri = _mat(k_rope, "k_rope", _BF16, dev)
    rows, d = ki[1], ki[3]
    if ki[2] != h or d != w - ROPE_DIM or vi[1:4] != ki[1:4] or ri[1:3] != (rows, ROPE_DIM):
        raise ValueError("q, k, v and k_rope do not match")
    n_seq = _device_len(q_start, "q_start") - 1
    args = (_dev(q, "q", _BF16, q.numel(), dev), ki[0], vi[0], ri[0], ki[4], ki[5], vi[4], vi[5], ri[3],
            _dev(q_start, "q_start", _I32, n_seq + 1, dev),
            _dev(kv_start, "kv_start", _I32, n_seq + 1, dev), n_seq, n, rows, h, d, scale,
            _out(out, n * h * d, dev), _kv_dtype(out), *_ws(workspace, dev), _status(d_status, dev))
    _check((_lib or lib()).omnitide_latent_chunk_attn(*args, _on(q, stream)),
           "omnitide_latent_chunk_attn")


def _device_len(t, name: str) -> int:
    if not isinstance(t, _T):
        raise TypeError(f"{name} must be a tensor")
    return t.numel()
