"""The paged cache made smaller, in bits and in tokens, behind the calls of ``attention.py``.

``qkv_append_q8``, ``attention_prefill_q8`` and ``attention_decode_q8`` are the attention
layer's calls over a cache of 8-bit codes (int8 or float8_e4m3fn) with a float32 scale for
each block of tokens and key head.  ``attention_weights`` adds the softmax weights that
queries place on the cached tokens to a running sum of each token and key head, over 16-bit
or 8-bit keys, and ``cache_evict`` keeps each sequence's heaviest tokens.  The C entry points
and their contract are in ``include/sls.h``.

A cache of codes is two tensors ``num_pages x page_size x kv_heads x head_dim``, its scales two
float32 tensors ``num_pages x (page_size / block) x kv_heads`` with blocks of 16, 32, 64 or 128
tokens; an element stands for code * scale.  Weights are a float32 tensor ``num_pages x kv_heads
x page_size``, zero where a page begins its life.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import Optional

import torch

import paper_2607_19368_gb300 as _sls

from . import attention as _at
from .attention import (Rope, _attention_rows, _cache, _call, _ints, _rows, _scratch,
                        _size_args, _weight)

__all__ = ["SLS_I8", "SLS_E4M3", "qkv_append_q8", "attention_prefill_q8", "attention_decode_q8",
           "attention_weights", "cache_evict"]

SLS_I8, SLS_E4M3 = 3, 4

_vp, _i64, _i32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float,
                              ctypes.c_size_t)

# name -> (restype, argtypes); structures go as packed bytes
EXPORTED = {
    "sls_qkv_append_q8": (_i32, [_vp, _vp, _vp, _i64, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp,
                                 _f32, _vp, _vp, _vp]),
    "sls_attention_prefill_q8_workspace_size": (_sz, [_i64, _i32, _vp, _vp, _i32]),
    "sls_attention_prefill_q8": (_i32, [_vp, _i64, _i32, _vp, _vp, _i32, _vp, _i32, _f32, _vp,
                                        _vp, _sz, _vp]),
    "sls_attention_decode_q8_workspace_size": (_sz, [_i32, _vp, _vp, _i32]),
    "sls_attention_decode_q8": (_i32, [_vp, _i32, _vp, _vp, _i32, _f32, _vp, _vp, _sz, _vp]),
    "sls_attention_weights_workspace_size": (_sz, [_i64, _i32, _vp, _vp, _i32]),
    "sls_attention_weights": (_i32, [_vp, _i64, _i32, _vp, _vp, _i32, _vp, _i32, _f32, _vp, _vp,
                                     _sz, _vp]),
    "sls_cache_evict": (_i32, [_vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp]),
}

_CODES8 = {torch.int8: SLS_I8, torch.float8_e4m3fn: SLS_E4M3}
_ANY = {**_at._CODES, **_CODES8}

# sls_kv_scales_t and sls_kv_weights_t in native layout
_SCALES = struct.Struct("@PPiqqq")
_WEIGHTS = struct.Struct("@Pqq")
_pack_scales, _pack_weights = _SCALES.pack, _WEIGHTS.pack


def _scales(k_scale, v_scale, pages, ps, H, dev):
    """(packed sls_kv_scales_t, block)"""
    shape = k_scale.shape
    if len(shape) != 3 or shape[0] != pages or shape[2] != H or shape[1] < 1 or ps % shape[1] \
            or k_scale.dtype != torch.float32 or k_scale.get_device() != dev:
        raise ValueError("k_scale, v_scale: float32 pages x (page_size / block) x kv_heads on the "
                         "cache's device")
    strides = k_scale.stride()
    if v_scale is None:
        vp = 0
    else:
        if v_scale.shape != shape or v_scale.dtype != torch.float32 \
                or v_scale.get_device() != dev or v_scale.stride() != strides:
            raise ValueError("k_scale, v_scale: two of one shape, strides, type and device")
        vp = v_scale.data_ptr()
    sp, sb, sh = strides
    # the stride of a dimension of one entry says nothing
    if shape[2] == 1:
        sh = 1
    if shape[1] == 1:
        sb = 1
    if pages == 1:
        sp = 1
    block = ps // shape[1]
    return _pack_scales(k_scale.data_ptr(), vp, block, sp, sb, sh), block


def _weights(weights, pages, ps, H, dev):
    if weights.shape != (pages, H, ps) or weights.dtype != torch.float32 \
            or weights.get_device() != dev or weights.stride(2) != 1:
        raise ValueError("weights: float32 pages x kv_heads x page_size on the cache's device, a "
                         "head's slots contiguous")
    sp, sh, _ = weights.stride()
    if H == 1:
        sh = ps
    if pages == 1:
        sp = H * sh
    return _pack_weights(weights.data_ptr(), sp, sh)


def _query(q):
    code = _at._CODES.get(q.dtype)
    if code is None:
        raise TypeError(f"unsupported query dtype {q.dtype} (bfloat16 or float16)")
    return code


# a workspace's size depends on these numbers alone (pointers that are never read stand in)
@functools.lru_cache(maxsize=256)
def _bytes(fn, dev, code, block, rest, cache) -> int:
    s = _pack_scales(256, 256, block, 1, 1, 1) if block else None
    c = _size_args(code, *cache)
    with torch.cuda.device(dev):
        lib = _sls.lib()
        if fn == "decode":
            return int(lib.sls_attention_decode_q8_workspace_size(rest[0], c, s, rest[1]))
        if fn == "prefill":
            return int(lib.sls_attention_prefill_q8_workspace_size(rest[0], rest[1], c, s, rest[2]))
        return int(lib.sls_attention_weights_workspace_size(rest[0], rest[1], c, s, rest[2]))


def qkv_append_q8(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cache_k: torch.Tensor,
                  cache_v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                  page_table: torch.Tensor, kv_lens: torch.Tensor,
                  cu_seqlens: Optional[torch.Tensor] = None,
                  positions: Optional[torch.Tensor] = None,
                  q_weight: Optional[torch.Tensor] = None,
                  k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  rope: Optional[Rope] = None,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``qkv_append`` into a cache of codes: q, k, v, out and the weights are bfloat16 or
    float16.  A block's scale is the least power of two that holds its tokens; a block that
    holds earlier tokens keeps its scale or, where a new token needs a larger one, has their
    codes rounded again.  Returns the queries (`out`, which may be q)."""
    dt = q.dtype
    dtype = _query(q)
    c, (n, ps, H, hd), _, dev, B, _ = _cache(cache_k, cache_v, page_table, kv_lens, _CODES8)
    s, _ = _scales(k_scale, v_scale, n, ps, H, dev)
    shape = q.shape
    if out is None:
        out = q.new_empty(shape)
    elif out.shape != shape:
        raise ValueError("out: the shape of q")
    T = shape[0]
    if k.shape[0] != T or v.shape[0] != T:
        raise ValueError("k and v: one row per token of q and key head")
    rq, ro = _rows("q", q, dt, 0, hd, dev), _rows("out", out, dt, 0, hd, dev)
    rk, rv = _rows("k", k, dt, H, hd, dev), _rows("v", v, dt, H, hd, dev)
    if cu_seqlens is None and T != B:
        raise ValueError("without cu_seqlens q has one token per sequence")
    # tensors keep their names: one that a caller makes for this call lives until it is enqueued
    cu = None if cu_seqlens is None else _ints("cu_seqlens", cu_seqlens, B + 1, dev)
    pos = None if positions is None else _ints("positions", positions, T, dev)
    wq = None if q_weight is None else _weight("q_weight", q_weight, dt, hd, dev)
    wk = None if k_weight is None else _weight("k_weight", k_weight, dt, hd, dev)
    if rope is not None and rope.inv_freq.get_device() != dev:
        raise ValueError("rope: frequencies on the cache's device")
    _call("sls_qkv_append_q8", dev, rq, rk, rv, T, shape[1], c, s, dtype, cu, pos, wq, wk, eps,
          None if rope is None else rope._c, ro)
    return out


def attention_prefill_q8(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                         k_scale: torch.Tensor, v_scale: torch.Tensor, page_table: torch.Tensor,
                         kv_lens: torch.Tensor, cu_seqlens: torch.Tensor, causal: bool = True,
                         scale: Optional[float] = None,
                         workspace: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``attention_prefill`` over a cache of codes; q (bfloat16 or float16) sets the type of the
    products and of the result.  The workspace holds the sequences' pages in that type, 4 bytes
    an element of keys and values."""
    dtype = _query(q)
    c, (n, ps, H, hd), dt, dev, B, cols = _cache(cache_k, cache_v, page_table, kv_lens, _CODES8)
    s, block = _scales(k_scale, v_scale, n, ps, H, dev)
    rq, ro, out, scale = _attention_rows(q, out, scale, q.dtype, hd, dev)
    cu = _ints("cu_seqlens", cu_seqlens, B + 1, dev)
    T, Hq, _ = q.shape
    nbytes = _bytes("prefill", dev, _CODES8[dt], block, (T, Hq, dtype), (H, hd, ps, n, B, cols))
    wp = 0
    if nbytes:
        workspace = _scratch(nbytes, workspace, q, dev)
        wp, nbytes = workspace.data_ptr(), workspace.numel()
    _call("sls_attention_prefill_q8", dev, rq, T, Hq, c, s, dtype, cu, causal, scale, ro, wp,
          nbytes)
    return out


def attention_decode_q8(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                        k_scale: torch.Tensor, v_scale: torch.Tensor, page_table: torch.Tensor,
                        kv_lens: torch.Tensor, scale: Optional[float] = None,
                        workspace: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``attention_decode`` over a cache of codes; q is bfloat16 or float16."""
    dtype = _query(q)
    c, (n, ps, H, hd), dt, dev, B, cols = _cache(cache_k, cache_v, page_table, kv_lens, _CODES8)
    s, block = _scales(k_scale, v_scale, n, ps, H, dev)
    rq, ro, out, scale = _attention_rows(q, out, scale, q.dtype, hd, dev)
    T, Hq, _ = q.shape
    if T != B:
        raise ValueError("q: one token per sequence")
    nbytes = _bytes("decode", dev, _CODES8[dt], block, (Hq, dtype), (H, hd, ps, n, B, cols))
    wp = 0
    if nbytes:
        workspace = _scratch(nbytes, workspace, q, dev)
        wp, nbytes = workspace.data_ptr(), workspace.numel()
    _call("sls_attention_decode_q8", dev, rq, Hq, c, s, dtype, scale, ro, wp, nbytes)
    return out


def attention_weights(q: torch.Tensor, cache_k: torch.Tensor, page_table: torch.Tensor,
                      kv_lens: torch.Tensor, weights: torch.Tensor,
                      cu_seqlens: Optional[torch.Tensor] = None,
                      k_scale: Optional[torch.Tensor] = None, causal: bool = True,
                      scale: Optional[float] = None,
                      workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Adds to `weights`, for every cached token and key head, the softmax weights that the
    queries (T x q_heads x head_dim, packed by cu_seqlens; None: one token per sequence) place
    on it, summed over the tokens and the head's query heads.  Rows see what they see in
    ``attention_prefill``: give the last few tokens of a prompt to let them alone vote.
    cache_k is of q's type, or codes with k_scale.  For few rows the workspace goes by the
    page table's width, up to 1 GiB.  Returns `weights`."""
    dtype = _query(q)
    c, (n, ps, H, hd), dt, dev, B, cols = _cache(cache_k, cache_k, page_table, kv_lens,
                                                 _ANY if k_scale is not None else _at._CODES)
    s, block = None, 0
    if k_scale is not None:
        if dt not in _CODES8:
            raise TypeError("k_scale goes with a cache of codes")
        s, block = _scales(k_scale, None, n, ps, H, dev)
    elif dt != q.dtype:
        raise TypeError("q and a 16-bit cache: one type")
    w = _weights(weights, n, ps, H, dev)
    rq = _rows("q", q, q.dtype, 0, hd, dev)
    T, Hq, _ = q.shape
    if cu_seqlens is None and T != B:
        raise ValueError("without cu_seqlens q has one token per sequence")
    # not by the tensor's own name: one made for this call must outlive the workspace's allocation
    cu = None if cu_seqlens is None else _ints("cu_seqlens", cu_seqlens, B + 1, dev)
    nbytes = _bytes("weights", dev, _ANY[dt], block, (T, Hq, dtype), (H, hd, ps, n, B, cols))
    wp = 0
    if nbytes:
        workspace = _scratch(nbytes, workspace, q, dev)
        wp, nbytes = workspace.data_ptr(), workspace.numel()
    _call("sls_attention_weights", dev, rq, T, Hq, c, s, dtype, cu, causal,
          hd ** -0.5 if scale is None else float(scale), w, wp, nbytes)
    return weights


def cache_evict(cache_k: torch.Tensor, cache_v: torch.Tensor, page_table: torch.Tensor,
                kv_lens: torch.Tensor, weights: torch.Tensor, keep: int, first: int = 0,
                last: int = 0, k_scale: Optional[torch.Tensor] = None,
                v_scale: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Cuts every sequence of more than `keep` tokens to `keep`: for each key head its first
    `first` and last `last` tokens and the others of the largest weights stay (equal ones: the
    lowest index) and move to the front in their order: keys, values, weights and, for codes,
    scales.  kv_lens is cut too, weights behind it are zeroed.  Returns the indices that
    stayed (B x kv_heads x keep int32, ascending, -1 past a shorter sequence's end).  Give
    later calls of ``qkv_append`` their positions: lengths no longer tell them.
    Layers that share kv_lens each want a copy of the lengths before the cut: over lengths
    that are cut already the call leaves a layer's cache as it is."""
    eight = k_scale is not None
    c, (n, ps, H, _), _, dev, B, _ = _cache(cache_k, cache_v, page_table, kv_lens,
                                            _CODES8 if eight else _at._CODES)
    if eight != (v_scale is not None):
        raise ValueError("k_scale, v_scale: both or none")
    s = _scales(k_scale, v_scale, n, ps, H, dev)[0] if eight else None
    w = _weights(weights, n, ps, H, dev)
    if keep < 0 or first < 0 or last < 0 or first + last > keep:
        raise ValueError("keep: at least first + last, none of them negative")
    kept = kv_lens.new_empty((B, H, keep))
    _call("sls_cache_evict", dev, c, s, w, keep, first, last, kept.data_ptr(),
          kv_lens.data_ptr())
    return kept
