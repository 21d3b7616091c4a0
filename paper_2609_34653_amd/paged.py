"""Thin Python binding of the paged-cache calls of libomnitide.so (include/omnitide_paged.h).

As in ``omnitide``: each function has the name of the C entry point it calls, checks its tensors,
passes the current HIP stream, and raises ``OmnitideError`` with the library's status code on
failure; every step of the computation runs in the HIP kernels.

Shapes: pools bf16 [n_pages, page_size, H_kv, d]; page_table int32 [n_seq, max_pages]; q_start
int32 [n_seq + 1]; ctx_len int32 [n_seq].  Queries, keys and values of new tokens are [tokens, heads,
d]; where a call takes row strides, parts of one fused projection (views whose heads are contiguous)
can be passed.  Tensors of one call are on one device, the current one unless ``stream`` is a
stream of theirs.
"""
from __future__ import annotations

import ctypes

import torch

from . import omnitide as ot
from .omnitide import (BF16, F32, ROPE_HALF, ROPE_INTERLEAVED, OmnitideError,  # noqa: F401
                       _buf, _check, _dev, _kv_dtype, _need, _out, _status, _stream)

ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_RAMP = 0, 1, 2, 3
E_PAGES = -19

EXPORTS = ("omnitide_rope_thetas", "omnitide_qk_norm_rope", "omnitide_paged_append",
           "omnitide_paged_chunk_attn", "omnitide_paged_chunk_attn_workspace_bytes",
           "omnitide_paged_decode_attn", "omnitide_paged_decode_workspace_bytes")

_P, _I, _SZ, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int64
_D, _F = ctypes.c_double, ctypes.c_float
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded HIP library with the paged calls declared."""
    global _lib
    if _lib is None:
        L = ot.lib()
        L.omnitide_rope_thetas.argtypes = [_D, _I, _I, _D, _D, _D, _D, _P]
        L.omnitide_qk_norm_rope.argtypes = [_P, _P, _I, _I, _I, _I, _I, _L, _L, _P, _P, _P, _F, _P,
                                            _I, _I, _F, _P, _P, _L, _L, _I, _P]
        L.omnitide_paged_append.argtypes = [_P, _P, _P, _I, _I, _I, _I, _I, _L, _L, _L, _P, _P, _I,
                                            _I, _P, _I, _P, _P, _I, _P, _P, _P, _F, _P, _I, _I, _F,
                                            _P, _L, _P, _P]
        L.omnitide_paged_chunk_attn.argtypes = [_P, _P, _P, _I, _I, _P, _I, _P, _P, _I, _I, _I, _I,
                                                _I, _F, _P, _I, _P, _SZ, _P, _P]
        L.omnitide_paged_decode_attn.argtypes = [_P, _P, _P, _I, _I, _P, _I, _P, _I, _I, _I, _I,
                                                 _I, _F, _P, _I, _P, _SZ, _P, _P]
        for name in ("omnitide_paged_chunk_attn_workspace_bytes",
                     "omnitide_paged_decode_workspace_bytes"):
            getattr(L, name).argtypes = [_I] * 6
            getattr(L, name).restype = _SZ
        for name in ("omnitide_rope_thetas", "omnitide_qk_norm_rope", "omnitide_paged_append",
                     "omnitide_paged_chunk_attn", "omnitide_paged_decode_attn"):
            getattr(L, name).restype = _I
        _lib = L
    return _lib


# ----------------------------------------------------------------------------- marshalling

def _on(t, stream):
    """The raw stream to launch on: `stream`, or the current one of t's device, which has to be the
    current device."""
    if stream is not None:
        return _stream(stream)
    dev = torch.cuda.current_device()
    if t.device.index != dev:
        raise ValueError(f"tensors on {t.device} while device {dev} is the current one")
    return torch._C._cuda_getCurrentRawStream(dev)


def _rows(t, name: str, dtypes):
    """(address, tokens, heads, d, row stride in elements) of [tokens, heads, d] with contiguous
    heads."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype} not in {list(dtypes)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, d]")
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if (d > 1 and s2 != 1) or (h > 1 and s1 != d):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t.data_ptr(), n, h, d, s0 if n > 1 else h * d


def _weight(w, name: str, dtype, d: int):
    return None if w is None else _dev(w, name, dtype, d)


def _theta(theta):
    """(address, rope_dims) of the host frequencies: a contiguous float64 CPU tensor or None."""
    if theta is None:
        return None, 0
    if not (isinstance(theta, torch.Tensor) and theta.dtype == torch.float64 and not theta.is_cuda
            and theta.dim() == 1 and theta.is_contiguous()):
        raise TypeError("theta must be a contiguous float64 CPU tensor [rope_dims / 2]")
    return theta.data_ptr(), 2 * theta.numel()


def _pools(k_pool, v_pool):
    """(k address, v address, n_pages, page_size, H_kv, d)."""
    if not (isinstance(k_pool, torch.Tensor) and k_pool.dim() == 4):
        raise ValueError("k_pool must be [n_pages, page_size, H_kv, d]")
    if not isinstance(v_pool, torch.Tensor) or v_pool.shape != k_pool.shape:
        raise ValueError("v_pool must have k_pool's shape")
    n = k_pool.numel()
    return (_dev(k_pool, "k_pool", _BF16, n), _dev(v_pool, "v_pool", _BF16, n), *k_pool.shape)


def _table(page_table, ctx_len):
    """(table address, max_pages, ctx_len address, n_seq)."""
    if not (isinstance(page_table, torch.Tensor) and page_table.dim() == 2):
        raise ValueError("page_table must be [n_seq, max_pages]")
    n_seq, max_pages = page_table.shape
    return (_dev(page_table, "page_table", _I32, n_seq * max_pages), max_pages,
            _dev(ctx_len, "ctx_len", _I32, n_seq), n_seq)


# ----------------------------------------------------------------------------------- calls

def omnitide_rope_thetas(rope_base, rope_dims, scaling=ROPE_PLAIN, factor=1.0, original_len=0.0,
                         ramp_slow=1.0, ramp_fast=32.0) -> torch.Tensor:
    """Rotary frequencies (float64, CPU, [rope_dims / 2]) for the calls below; a host function."""
    n = max(0, int(rope_dims) // 2)
    theta = torch.empty(max(1, n), dtype=torch.float64)
    _check(lib().omnitide_rope_thetas(float(rope_base), int(rope_dims), int(scaling), float(factor),
                                      float(original_len), float(ramp_slow), float(ramp_fast),
                                      theta.data_ptr() if n <= 64 else None),
           "omnitide_rope_thetas")
    return theta


def omnitide_qk_norm_rope(q, k, pos, q_out, k_out, theta=None, rope_style=ROPE_HALF, magnitude=1.0,
                          q_weight=None, k_weight=None, eps=1e-6, stream=None):
    """Per-head RMS norm (weights given) and rotation (theta given) of q and k into q_out and k_out
    (all [tokens, heads, d]; an output may be its input).  q or k may be None, with its output."""
    first = q if q is not None else k
    if first is None:
        raise ValueError("q or k must be given")
    dt, out = first.dtype, (q_out if q is not None else k_out).dtype
    qi = qo = ki = ko = (None, 0, 0, 0, 0)
    if q is not None:
        qi, qo = _rows(q, "q", (_BF16, _F32)), _rows(q_out, "q_out", (_BF16, _F32))
        if q_out.shape != q.shape:
            raise ValueError("q_out must have q's shape")
    if k is not None:
        ki, ko = _rows(k, "k", (dt,)), _rows(k_out, "k_out", (out,))
        if k_out.shape != k.shape:
            raise ValueError("k_out must have k's shape")
    _, n, _, d, _ = qi if q is not None else ki
    if k is not None and (ki[1] != n or ki[3] != d):
        raise ValueError("k does not match q")
    th, dims = _theta(theta)
    _check(lib().omnitide_qk_norm_rope(
        qi[0], ki[0], _kv_dtype(first), n, qi[2], ki[2], d, qi[4], ki[4],
        None if pos is None else _dev(pos, "pos", _I32, n), _weight(q_weight, "q_weight", dt, d),
        _weight(k_weight, "k_weight", dt, d), float(eps), th, dims, int(rope_style),
        float(magnitude), qo[0], ko[0], qo[4], ko[4], BF16 if out == _BF16 else F32,
        _on(first, stream)), "omnitide_qk_norm_rope")


def omnitide_paged_append(k, v, k_pool, v_pool, page_table, q_start, ctx_len, pos=None, theta=None,
                          rope_style=ROPE_HALF, magnitude=1.0, k_weight=None, eps=1e-6, q=None,
                          q_out=None, q_weight=None, d_status=None, stream=None):
    """The new tokens' k (normed, rotated) and v into the pages; q into q_out (bf16) if given."""
    dt = k.dtype
    ki, vi = _rows(k, "k", (_BF16, _F32)), _rows(v, "v", (dt,))
    if v.shape != k.shape:
        raise ValueError("v must have k's shape")
    n, d = ki[1], ki[3]
    qi = qo = (None, 0, 0, 0, 0)
    if q is not None or q_out is not None:
        qi, qo = _rows(q, "q", (dt,)), _rows(q_out, "q_out", (_BF16,))
        if qi[1] != n or qi[3] != d or q_out.shape != q.shape:
            raise ValueError("q, q_out and k do not match")
    kp, vp, n_pages, page, hkv, dp = _pools(k_pool, v_pool)
    if hkv != ki[2] or dp != d:
        raise ValueError("the pools do not match k")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len)
    th, dims = _theta(theta)
    _check(lib().omnitide_paged_append(
        ki[0], vi[0], qi[0], _kv_dtype(k), n, qi[2], hkv, d, ki[4], vi[4], qi[4], kp, vp, n_pages,
        page, tab, max_pages, _dev(q_start, "q_start", _I32, n_seq + 1), ctx, n_seq,
        None if pos is None else _dev(pos, "pos", _I32, n), _weight(k_weight, "k_weight", dt, d),
        _weight(q_weight, "q_weight", dt, d), float(eps), th, dims, int(rope_style),
        float(magnitude), qo[0], qo[4], _status(d_status), _on(k, stream)),
        "omnitide_paged_append")


def omnitide_paged_chunk_attn_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads, n_kv_heads,
                                              head_dim) -> int:
    return int(lib().omnitide_paged_chunk_attn_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads,
                                                               n_kv_heads, head_dim))


def _ws(workspace):
    return (None, 0) if workspace is None else (_buf(workspace), workspace.numel())


def omnitide_paged_chunk_attn(q, k_pool, v_pool, page_table, q_start, ctx_len, scale, out,
                              workspace=None, d_status=None, stream=None):
    """q [tokens, H_q, d] bf16 of a ragged batch of chunks; out float32 or bf16 like q."""
    if q.dim() != 3:
        raise ValueError("q must be [tokens, H_q, d]")
    n, hq, d = q.shape
    kp, vp, n_pages, page, hkv, dp = _pools(k_pool, v_pool)
    if dp != d:
        raise ValueError("the pools do not match q")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len)
    args = (_dev(q, "q", _BF16, q.numel()), kp, vp, n_pages, page, tab, max_pages,
            _dev(q_start, "q_start", _I32, n_seq + 1), ctx, n_seq, n, hq, hkv, d, float(scale),
            _out(out, q.numel()), _kv_dtype(out), *_ws(workspace), _status(d_status))
    _check(lib().omnitide_paged_chunk_attn(*args, _on(q, stream)), "omnitide_paged_chunk_attn")


def omnitide_paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads, n_kv_heads,
                                          head_dim) -> int:
    return int(lib().omnitide_paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads,
                                                           n_kv_heads, head_dim))


def omnitide_paged_decode_attn(q, k_pool, v_pool, page_table, ctx_len, scale, out, workspace=None,
                               d_status=None, stream=None):
    """q [n_seq, n_q, H_q, d] bf16 (the last n_q tokens of each sequence); out float32 or bf16 like
    q.  A sequence with ctx_len 0 is idle: zeros."""
    if q.dim() != 4:
        raise ValueError("q must be [n_seq, n_q, H_q, d]")
    n_seq, nq, hq, d = q.shape
    kp, vp, n_pages, page, hkv, dp = _pools(k_pool, v_pool)
    tab, max_pages, ctx, ns = _table(page_table, ctx_len)
    if dp != d or ns != n_seq:
        raise ValueError("the pools or the table do not match q")
    args = (_dev(q, "q", _BF16, q.numel()), kp, vp, n_pages, page, tab, max_pages, ctx, n_seq, nq,
            hq, hkv, d, float(scale), _out(out, q.numel()), _kv_dtype(out), *_ws(workspace),
            _status(d_status))
    _check(lib().omnitide_paged_decode_attn(*args, _on(q, stream)), "omnitide_paged_decode_attn")
