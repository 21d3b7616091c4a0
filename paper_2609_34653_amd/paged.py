"""Thin Python binding of the paged-cache calls of libomnitide.so (include/omnitide_paged.h).

As in ``omnitide``: each function has the name of the C entry point it calls, checks its tensors,
passes the current HIP stream, and raises ``OmnitideError`` with the library's status code on
failure; every step of the computation runs in the HIP kernels.

Shapes: pools bf16 [n_pages, page_size, H_kv, d]; page_table int32 [n_seq, max_pages]; q_start
int32 [n_seq + 1]; ctx_len int32 [n_seq].  Queries, keys and values of new tokens are [tokens, heads,
d]; where a call takes row strides, parts of one fused projection (views whose heads are contiguous)
can be passed.  Tensors of one call, and its ``stream`` if given, belong to the current device: every
tensor is checked, and the stream where it knows its device (a bare handle does not).
"""
from __future__ import annotations

import ctypes

import torch

from . import omnitide as ot
from .omnitide import (BF16, F32, ROPE_HALF, ROPE_INTERLEAVED, OmnitideError,  # noqa: F401
                       _check, _kv_dtype, _need, _stream)

ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_RAMP = 0, 1, 2, 3
E_PAGES = -19

EXPORTS = ("omnitide_rope_thetas", "omnitide_qk_norm_rope", "omnitide_paged_append",
           "omnitide_paged_chunk_attn", "omnitide_paged_chunk_attn_workspace_bytes",
           "omnitide_paged_decode_attn", "omnitide_paged_decode_workspace_bytes")

_P, _I, _SZ, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int64
_D, _F = ctypes.c_double, ctypes.c_float
_T, _BF16, _F32, _I32 = torch.Tensor, torch.bfloat16, torch.float32, torch.int32

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
    """The raw stream to launch on: `stream`, or the current one; t has to be on the current
    device, and so has a stream object."""
    dev = torch._C._cuda_getDevice()
    if t.get_device() != dev:
        raise ValueError(f"tensors on {t.device} while device {dev} is the current one")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"a stream of {stream.device} while device {dev} is the current one")
    return _stream(stream)


# As in ``omnitide``, a tensor in order takes one short path; a call passes up to 15 tensors, and a step
# of single tokens is bound by its calls' marshalling.  `dev` is the number of the first tensor's device
# (_on asks for the current one there).

def _device(t, name: str) -> int:
    if not isinstance(t, _T):
        raise TypeError(f"{name} must be a tensor")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a device tensor")
    return dev


def _same(t, name: str, dev: int):
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on device {dev}")


def _dev(t, name: str, dtype, numel: int, dev: int) -> int:
    """Address of a contiguous tensor of `dtype` and `numel` elements on device `dev`."""
    if not (type(t) is _T and t.dtype is dtype and t.get_device() == dev and t.is_contiguous()
            and t.numel() == numel):
        _need(t, name, (dtype,), numel)
        _same(t, name, dev)
    return t.data_ptr()


def _out(out, numel: int, dev: int) -> int:
    """Address of a float32 or bf16 output."""
    if not (type(out) is _T and (out.dtype is _F32 or out.dtype is _BF16)
            and out.get_device() == dev and out.is_contiguous() and out.numel() == numel):
        _need(out, "out", (_F32, _BF16), numel)
        _same(out, "out", dev)
    return out.data_ptr()


def _status(t, dev: int):
    return None if t is None else _dev(t, "d_status", _I32, 1, dev)


def _ws(t, dev: int):
    """(address, bytes) of the workspace."""
    if t is None:
        return None, 0
    if not (type(t) is _T and t.dtype is torch.uint8 and t.get_device() == dev
            and t.is_contiguous()):
        _need(t, "workspace", (torch.uint8,))
        _same(t, "workspace", dev)
    return t.data_ptr(), t.numel()


def _rows(t, name: str, dtype, dev: int):
    """(address, tokens, heads, d, row stride in elements) of [tokens, heads, d] of dtype with
    contiguous heads."""
    if not (type(t) is _T and t.dtype is dtype and t.get_device() == dev and t.dim() == 3):
        if not isinstance(t, _T):
            raise TypeError(f"{name} must be a tensor")
        if t.dtype is not dtype:
            raise TypeError(f"{name}: dtype {t.dtype} is not {dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        _same(t, name, dev)
        if t.dim() != 3:
            raise ValueError(f"{name} must be [tokens, heads, d]")
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if (s2 == 1 or d == 1) and (s1 == d or h == 1):
        return t.data_ptr(), n, h, d, s0 if n > 1 else h * d
    raise ValueError(f"{name}: the heads of a token must be contiguous")


def _float_type(t, name: str):
    if not isinstance(t, _T):
        raise TypeError(f"{name} must be a tensor")
    if t.dtype is not _BF16 and t.dtype is not _F32:
        raise TypeError(f"{name}: dtype {t.dtype} is not bfloat16 or float32")
    return t.dtype


def _theta(theta):
    """(address, rope_dims) of the host frequencies: a contiguous float64 CPU tensor or None."""
    if theta is None:
        return None, 0
    if not (isinstance(theta, _T) and theta.dtype is torch.float64 and not theta.is_cuda
            and theta.dim() == 1 and theta.is_contiguous()):
        raise TypeError("theta must be a contiguous float64 CPU tensor [rope_dims / 2]")
    return theta.data_ptr(), 2 * theta.numel()


def _pools(k_pool, v_pool, dev: int):
    """(k address, v address, n_pages, page_size, H_kv, d)."""
    if type(k_pool) is _T and type(v_pool) is _T:
        shape = k_pool.shape
        if (len(shape) == 4 and v_pool.shape == shape and k_pool.dtype is _BF16
                and v_pool.dtype is _BF16 and k_pool.get_device() == dev
                and v_pool.get_device() == dev
                and k_pool.is_contiguous() and v_pool.is_contiguous()):
            return (k_pool.data_ptr(), v_pool.data_ptr(), *shape)
    if not (isinstance(k_pool, _T) and k_pool.dim() == 4):
        raise ValueError("k_pool must be [n_pages, page_size, H_kv, d]")
    shape = k_pool.shape
    if not isinstance(v_pool, _T) or v_pool.shape != shape:
        raise ValueError("v_pool must have k_pool's shape")
    n = k_pool.numel()
    return (_dev(k_pool, "k_pool", _BF16, n, dev), _dev(v_pool, "v_pool", _BF16, n, dev), *shape)


def _table(page_table, ctx_len, dev: int):
    """(table address, max_pages, ctx_len address, n_seq)."""
    if not (isinstance(page_table, _T) and page_table.dim() == 2):
        raise ValueError("page_table must be [n_seq, max_pages]")
    n_seq, max_pages = page_table.shape
    if (type(page_table) is _T and page_table.dtype is _I32 and page_table.get_device() == dev
            and page_table.is_contiguous()):
        at = page_table.data_ptr()
    else:
        at = _dev(page_table, "page_table", _I32, n_seq * max_pages, dev)
    return at, max_pages, _dev(ctx_len, "ctx_len", _I32, n_seq, dev), n_seq


# ----------------------------------------------------------------------------------- calls

def omnitide_rope_thetas(rope_base, rope_dims, scaling=ROPE_PLAIN, factor=1.0, original_len=0.0,
                         ramp_slow=1.0, ramp_fast=32.0) -> torch.Tensor:
    """Rotary frequencies (float64, CPU, [rope_dims / 2]) for the calls below; a host function."""
    dims = int(rope_dims)
    theta = torch.empty(max(1, min(dims, 128) // 2), dtype=torch.float64)   # the library refuses others
    _check(lib().omnitide_rope_thetas(float(rope_base), max(-1, min(dims, 1 << 20)), int(scaling),
                                      float(factor), float(original_len), float(ramp_slow),
                                      float(ramp_fast), theta.data_ptr()), "omnitide_rope_thetas")
    return theta


def omnitide_qk_norm_rope(q, k, pos, q_out, k_out, theta=None, rope_style=ROPE_HALF, magnitude=1.0,
                          q_weight=None, k_weight=None, eps=1e-6, stream=None):
    """Per-head RMS norm (weights given) and rotation (theta given) of q and k into q_out and k_out
    (all [tokens, heads, d]; an output may be its input).  q or k may be None, with its output."""
    first, out = (q, q_out) if q is not None else (k, k_out)
    if first is None:
        raise ValueError("q or k must be given")
    dt, odt = _float_type(first, "q or k"), _float_type(out, "q_out or k_out")
    dev = _device(first, "q or k")
    qi = qo = ki = ko = (None, 0, 0, 0, 0)
    if q is not None:
        qi, qo = _rows(q, "q", dt, dev), _rows(q_out, "q_out", odt, dev)
        if qi[1:4] != qo[1:4]:
            raise ValueError("q_out must have q's shape")
    if k is not None:
        ki, ko = _rows(k, "k", dt, dev), _rows(k_out, "k_out", odt, dev)
        if ki[1:4] != ko[1:4]:
            raise ValueError("k_out must have k's shape")
        if q is not None and (ki[1] != qi[1] or ki[3] != qi[3]):
            raise ValueError("k does not match q")
    n, d = (qi if q is not None else ki)[1:4:2]
    th, dims = _theta(theta)
    _check((_lib or lib()).omnitide_qk_norm_rope(
        qi[0], ki[0], BF16 if dt is _BF16 else F32, n, qi[2], ki[2], d, qi[4], ki[4],
        None if pos is None else _dev(pos, "pos", _I32, n, dev),
        None if q_weight is None else _dev(q_weight, "q_weight", dt, d, dev),
        None if k_weight is None else _dev(k_weight, "k_weight", dt, d, dev), eps, th, dims, rope_style,
        magnitude, qo[0], ko[0], qo[4], ko[4], BF16 if odt is _BF16 else F32, _on(first, stream)),
        "omnitide_qk_norm_rope")


def omnitide_paged_append(k, v, k_pool, v_pool, page_table, q_start, ctx_len, pos=None, theta=None,
                          rope_style=ROPE_HALF, magnitude=1.0, k_weight=None, eps=1e-6, q=None,
                          q_out=None, q_weight=None, d_status=None, stream=None):
    """The new tokens' k (normed, rotated) and v into the pages; q into q_out (bf16) if given."""
    dt = _float_type(k, "k")
    dev = _device(k, "k")
    ki, vi = _rows(k, "k", dt, dev), _rows(v, "v", dt, dev)
    n, hkv, d = ki[1:4]
    if vi[1:4] != (n, hkv, d):
        raise ValueError("v must have k's shape")
    qi = qo = (None, 0, 0, 0, 0)
    if q is not None or q_out is not None:
        qi, qo = _rows(q, "q", dt, dev), _rows(q_out, "q_out", _BF16, dev)
        if qi[1] != n or qi[3] != d or qi[1:4] != qo[1:4]:
            raise ValueError("q, q_out and k do not match")
    kp, vp, n_pages, page, hp, dp = _pools(k_pool, v_pool, dev)
    if hp != hkv or dp != d:
        raise ValueError("the pools do not match k")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    th, dims = _theta(theta)
    _check((_lib or lib()).omnitide_paged_append(
        ki[0], vi[0], qi[0], BF16 if dt is _BF16 else F32, n, qi[2], hkv, d, ki[4], vi[4], qi[4], kp,
        vp, n_pages, page, tab, max_pages, _dev(q_start, "q_start", _I32, n_seq + 1, dev), ctx,
        n_seq, None if pos is None else _dev(pos, "pos", _I32, n, dev),
        None if k_weight is None else _dev(k_weight, "k_weight", dt, d, dev),
        None if q_weight is None else _dev(q_weight, "q_weight", dt, d, dev), eps, th, dims,
        rope_style, magnitude, qo[0], qo[4], _status(d_status, dev), _on(k, stream)),
        "omnitide_paged_append")


def omnitide_paged_chunk_attn_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads, n_kv_heads,
                                              head_dim) -> int:
    return int(lib().omnitide_paged_chunk_attn_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads,
                                                               n_kv_heads, head_dim))


def omnitide_paged_chunk_attn(q, k_pool, v_pool, page_table, q_start, ctx_len, scale, out,
                              workspace=None, d_status=None, stream=None):
    """q [tokens, H_q, d] bf16 of a ragged batch of chunks; out float32 or bf16 like q."""
    dev = _device(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, H_q, d]")
    n, hq, d = q.shape
    kp, vp, n_pages, page, hkv, dp = _pools(k_pool, v_pool, dev)
    if dp != d:
        raise ValueError("the pools do not match q")
    tab, max_pages, ctx, n_seq = _table(page_table, ctx_len, dev)
    args = (_dev(q, "q", _BF16, q.numel(), dev), kp, vp, n_pages, page, tab, max_pages,
            _dev(q_start, "q_start", _I32, n_seq + 1, dev), ctx, n_seq, n, hq, hkv, d, scale,
            _out(out, q.numel(), dev), _kv_dtype(out), *_ws(workspace, dev),
            _status(d_status, dev))
    _check((_lib or lib()).omnitide_paged_chunk_attn(*args, _on(q, stream)),
           "omnitide_paged_chunk_attn")


def omnitide_paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads, n_kv_heads,
                                          head_dim) -> int:
    return int(lib().omnitide_paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads,
                                                           n_kv_heads, head_dim))


def omnitide_paged_decode_attn(q, k_pool, v_pool, page_table, ctx_len, scale, out, workspace=None,
                               d_status=None, stream=None):
    """q [n_seq, n_q, H_q, d] bf16 (the last n_q tokens of each sequence); out float32 or bf16 like
    q.  A sequence with ctx_len 0 is idle: zeros."""
    dev = _device(q, "q")
    if q.dim() != 4:
        raise ValueError("q must be [n_seq, n_q, H_q, d]")
    n_seq, nq, hq, d = q.shape
    kp, vp, n_pages, page, hkv, dp = _pools(k_pool, v_pool, dev)
    tab, max_pages, ctx, ns = _table(page_table, ctx_len, dev)
    if dp != d or ns != n_seq:
        raise ValueError("the pools or the table do not match q")
    args = (_dev(q, "q", _BF16, q.numel(), dev), kp, vp, n_pages, page, tab, max_pages, ctx, n_seq,
            nq, hq, hkv, d, scale, _out(out, q.numel(), dev), _kv_dtype(out), *_ws(workspace, dev),
            _status(d_status, dev))
    _check((_lib or lib()).omnitide_paged_decode_attn(*args, _on(q, stream)),
           "omnitide_paged_decode_attn")
