"""Attention over the macro-tokens: the calls that follow the compression pass
(prefill of the compressed prompt at the macro-tokens' positions, and decoding
behind it) over one paged cache of keys and values.

``qkv_append`` norms and rotates new queries and keys and appends keys and
values, ``attention_prefill`` is the attention of packed prompts,
``attention_decode`` that of one token per sequence; ``Rope`` holds the rotation's
frequencies.  The C entry points and their contract are in ``include/sls.h``.

The cache is two tensors ``num_pages x page_size x kv_heads x head_dim`` (bfloat16
or float16); ``page_table`` (B x max_pages int32) lists every sequence's pages and
``kv_lens`` (B int32) counts its cached tokens, new ones included.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from typing import Optional

import torch

import paper_2607_19368_gb300 as _sls

__all__ = ["SLS_F16", "Rope", "qkv_append", "attention_prefill", "attention_decode",
           "attention_status"]

SLS_F16 = 2

_vp, _i64, _i32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float,
                              ctypes.c_size_t)

# name -> (restype, argtypes); the attention part of include/sls.h.  Structures go as
# packed bytes (or byref of a ctypes structure).
EXPORTED = {
    "sls_qkv_append": (_i32, [_vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp,
                              _vp]),
    "sls_attention_prefill_workspace_size": (_sz, [_i64, _i32, _vp]),
    "sls_attention_prefill": (_i32, [_vp, _i64, _i32, _vp, _vp, _i32, _f32, _vp, _vp, _sz, _vp]),
    "sls_attention_decode_workspace_size": (_sz, [_i32, _vp]),
    "sls_attention_decode": (_i32, [_vp, _i32, _vp, _f32, _vp, _vp, _sz, _vp]),
    "sls_attention_status": (_i32, [_vp]),
}

_CODES = {torch.bfloat16: 1, torch.float16: SLS_F16}

# sls_kv_cache_t, sls_rows_t and sls_rope_t in native layout: the calls are a few
# microseconds of work on the GPU at their smallest, and packing is the cheapest way to
# hand a structure over
_CACHE = struct.Struct("@PPiiiiqqqqPqiPq")
_ROWS = struct.Struct("@Pqq")
_ROPE = struct.Struct("@Piif")
_pack_cache, _pack_rows = _CACHE.pack, _ROWS.pack
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


class Rope:
    """The rotation by position: pair i of a head turns by the angle
    ``position * inv_freq[i]`` (a float32 CUDA tensor, one entry per pair), its
    elements being i and pairs + i, or 2 i and 2 i + 1 when `interleaved`;
    `scale` multiplies the rotated part.  Elements past 2 * pairs stay as they
    are.  ``Rope.make`` forms the frequencies."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, scale: float = 1.0):
        if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_cuda:
            raise ValueError("inv_freq: a one-dimensional float32 CUDA tensor")
        self.inv_freq = inv_freq.contiguous()
        self.interleaved = bool(interleaved)
        self.scale = float(scale)
        self._c = _ROPE.pack(self.inv_freq.data_ptr(), self.inv_freq.numel(),
                             int(self.interleaved), self.scale)

    @classmethod
    def make(cls, rot_dim: int, base: float = 10000.0, interleaved: bool = False,
             factor: float = 1.0, original_length: Optional[int] = None,
             slow_turns: float = 1.0, fast_turns: float = 32.0, scale: float = 1.0,
             device="cuda") -> "Rope":
        """Frequencies base^(-2 i / rot_dim).  `factor` > 1 stretches the context:
        every frequency is divided by it (positions interpolated), or, with
        `original_length`, only those that turn less than `slow_turns` times over
        that length, with a linear blend in the number of turns up to
        `fast_turns`, from which a frequency is kept."""
        if rot_dim < 2 or rot_dim % 2:
            raise ValueError("rot_dim: a positive even number")
        if factor < 1.0:
            raise ValueError("factor: at least 1")
        i = torch.arange(rot_dim // 2, dtype=torch.float64)
        f = float(base) ** (-2.0 * i / rot_dim)
        if factor > 1.0:
            keep = torch.zeros_like(f)
            if original_length is not None:
                turns = original_length * f / (2.0 * math.pi)
                keep = ((turns - slow_turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
            f = f * (keep + (1.0 - keep) / factor)
        return cls(f.float().to(device), interleaved=interleaved, scale=scale)


def _rows(name: str, t: torch.Tensor, dtype, heads: int, head_dim: int, dev: int) -> bytes:
    shape = t.shape
    if len(shape) != 3 or shape[2] != head_dim or t.dtype != dtype or t.get_device() != dev \
            or (heads and shape[1] != heads):
        raise ValueError(f"{name}: tokens x {heads or 'heads'} x {head_dim} of {dtype} on the "
                         "cache's device")
    st, sh, se = t.stride()
    if se != 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    # the stride of a dimension of one entry says nothing
    if shape[1] == 1:
        sh = head_dim
    if shape[0] <= 1:
        st = sh * shape[1]
    return _pack_rows(t.data_ptr(), st, sh)


def _ints(name: str, t: torch.Tensor, n: int, dev: int) -> int:
    if t.dtype != torch.int32 or t.shape != (n,) or not t.is_contiguous() \
            or t.get_device() != dev:
        raise ValueError(f"{name}: {n} contiguous int32 entries on the cache's device")
    return t.data_ptr()


def _cache(cache_k, cache_v, page_table, kv_lens):
    """(packed sls_kv_cache_t, shape, dtype, device index, batch, page table columns)"""
    dt, shape, dev = cache_k.dtype, cache_k.shape, cache_k.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise TypeError(f"unsupported attention dtype {dt} (bfloat16 or float16)")
    strides = cache_k.stride()
    if dev < 0 or len(shape) != 4 or cache_v.shape != shape or cache_v.dtype != dt \
            or cache_v.get_device() != dev or strides[3] != 1 or cache_v.stride() != strides:
        raise ValueError("cache_k, cache_v: pages x page_size x kv_heads x head_dim on one GPU, "
                         "of equal strides, the elements of a head contiguous")
    table = page_table.shape
    if len(table) != 2 or page_table.dtype != torch.int32 or page_table.get_device() != dev:
        raise ValueError("page_table: B x max_pages int32 on the cache's device")
    B, cols = table
    ld, se = page_table.stride()
    if B <= 1:
        ld = cols
    if (se != 1 and cols > 1) or ld < cols:
        raise ValueError("page_table: contiguous rows that do not overlap")
    lens = _ints("kv_lens", kv_lens, B, dev)
    n, ps, H, hd = shape
    sp, ss, sh, _ = strides
    if H == 1:
        sh = hd
    if n == 1:
        sp = ps * max(ss, sh * H)
    return (_pack_cache(cache_k.data_ptr(), cache_v.data_ptr(), code, H, hd, ps, n, sp, ss, sh,
                        page_table.data_ptr(), ld, cols, lens, B),
            shape, dt, dev, B, cols)


def _weight(name: str, w: Optional[torch.Tensor], dtype, head_dim: int, dev: int):
    if w is None:
        return None
    if w.dtype != dtype or w.shape != (head_dim,) or not w.is_contiguous() \
            or w.get_device() != dev:
        raise ValueError(f"{name}: {head_dim} contiguous elements of {dtype} on the cache's device")
    return w.data_ptr()


def _call(fn: str, dev: int, *args):
    """A C call on the current stream of the tensors' device, which is made current: the
    library launches on the current one."""
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return _call(fn, dev, *args)
    st = getattr(_sls._lib or _sls.lib(), fn)(*args, _raw_stream(dev))
    if st != 0:
        _sls._check(fn, st)
    if _sls._CHECK_STATUS:
        st = attention_status(dev)
        if st != 0:
            raise _sls.SLSError(fn + " (device status)", st,
                                _sls.lib().sls_status_string(st).decode())


def qkv_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cache_k: torch.Tensor,
               cache_v: torch.Tensor, page_table: torch.Tensor, kv_lens: torch.Tensor,
               cu_seqlens: Optional[torch.Tensor] = None,
               positions: Optional[torch.Tensor] = None,
               q_weight: Optional[torch.Tensor] = None,
               k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
               rope: Optional[Rope] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm of queries and keys for each head (root mean square over head_dim,
    times q_weight / k_weight; skipped where the weight is None), rotation by
    `positions` (T int32; the cache index when None) if `rope` is given, and
    keys and values appended to the cache.  q is T x q_heads x head_dim, k and v
    T x kv_heads x head_dim (any token and head strides that are multiples of 8);
    cu_seqlens packs the new tokens (B + 1 int32; None: one token per sequence).
    kv_lens counts the new tokens.  Returns the queries (`out`, which may be q)."""
    c, (_, _, H, hd), dt, dev, B, _ = _cache(cache_k, cache_v, page_table, kv_lens)
    shape = q.shape
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != shape:
        raise ValueError("out: the shape of q")
    T = shape[0]
    if k.shape[0] != T or v.shape[0] != T:
        raise ValueError("k and v: one row per token of q and key head")
    rq, ro = _rows("q", q, dt, 0, hd, dev), _rows("out", out, dt, 0, hd, dev)
    rk, rv = _rows("k", k, dt, H, hd, dev), _rows("v", v, dt, H, hd, dev)
    if cu_seqlens is not None:
        cu_seqlens = _ints("cu_seqlens", cu_seqlens, B + 1, dev)
    elif T != B:
        raise ValueError("without cu_seqlens q has one token per sequence")
    if positions is not None:
        positions = _ints("positions", positions, T, dev)
    if q_weight is not None:
        q_weight = _weight("q_weight", q_weight, dt, hd, dev)
    if k_weight is not None:
        k_weight = _weight("k_weight", k_weight, dt, hd, dev)
    if rope is not None and rope.inv_freq.get_device() != dev:
        raise ValueError("rope: frequencies on the cache's device")
    _call("sls_qkv_append", dev, rq, rk, rv, T, shape[1], c, cu_seqlens, positions, q_weight,
          k_weight, eps, None if rope is None else rope._c, ro)
    return out


def _attention_rows(q, out, scale, dt, hd, dev):
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape:
        raise ValueError("out: the shape of q")
    return (_rows("q", q, dt, 0, hd, dev), _rows("out", out, dt, 0, hd, dev), out,
            hd ** -0.5 if scale is None else float(scale))


def _scratch(nbytes: int, workspace: Optional[torch.Tensor], q: torch.Tensor, dev: int):
    """A caller's workspace (a uint8 tensor) or one for this call."""
    if workspace is None:
        return q.new_empty(nbytes, dtype=torch.uint8)
    if workspace.get_device() != dev or workspace.dtype != torch.uint8 \
            or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous uint8 tensor on the cache's device")
    return workspace


# a workspace's size depends on these numbers alone (pointers that are never read stand
# in for the cache's)
def _size_args(code, H, hd, ps, n, B, cols):
    return _pack_cache(256, 256, code, H, hd, ps, n, ps * H * hd, H * hd, hd, 256, cols, cols,
                       256, B)


@functools.lru_cache(maxsize=256)
def _decode_bytes(dev, Hq, *cache) -> int:
    with torch.cuda.device(dev):
        return int(_sls.lib().sls_attention_decode_workspace_size(Hq, _size_args(*cache)))


@functools.lru_cache(maxsize=256)
def _prefill_bytes(dev, T, Hq, *cache) -> int:
    with torch.cuda.device(dev):
        return int(_sls.lib().sls_attention_prefill_workspace_size(T, Hq, _size_args(*cache)))


def attention_prefill(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                      page_table: torch.Tensor, kv_lens: torch.Tensor, cu_seqlens: torch.Tensor,
                      causal: bool = True, scale: Optional[float] = None,
                      workspace: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Softmax attention of packed new tokens (q: T x q_heads x head_dim, packed by
    cu_seqlens) over the cache that holds their keys and values: token i of a
    sequence with n new and kv_lens tokens sees the cache up to its own index
    kv_lens - n + i (causal) or all of it.  scale defaults to head_dim^-0.5.
    Returns q's shape; rows that see no key are zero."""
    c, (n, ps, H, hd), dt, dev, B, cols = _cache(cache_k, cache_v, page_table, kv_lens)
    rq, ro, out, scale = _attention_rows(q, out, scale, dt, hd, dev)
    cu = _ints("cu_seqlens", cu_seqlens, B + 1, dev)
    T, Hq, _ = q.shape
    nbytes = _prefill_bytes(dev, T, Hq, _CODES[dt], H, hd, ps, n, B, cols)
    wp = 0
    if nbytes:
        workspace = _scratch(nbytes, workspace, q, dev)
        wp, nbytes = workspace.data_ptr(), workspace.numel()
    _call("sls_attention_prefill", dev, rq, T, Hq, c, cu, causal, scale, ro, wp, nbytes)
    return out


def attention_decode(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                     page_table: torch.Tensor, kv_lens: torch.Tensor,
                     scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One token per sequence (q: B x q_heads x head_dim) over all kv_lens tokens of
    its sequence.  Returns q's shape; a sequence of length 0 gives zeros."""
    c, (n, ps, H, hd), dt, dev, B, cols = _cache(cache_k, cache_v, page_table, kv_lens)
    rq, ro, out, scale = _attention_rows(q, out, scale, dt, hd, dev)
    T, Hq, _ = q.shape
    if T != B:
        raise ValueError("q: one token per sequence")
    nbytes = _decode_bytes(dev, Hq, _CODES[dt], H, hd, ps, n, B, cols)
    wp = 0
    if nbytes:
        workspace = _scratch(nbytes, workspace, q, dev)
        wp, nbytes = workspace.data_ptr(), workspace.numel()
    _call("sls_attention_decode", dev, rq, Hq, c, scale, ro, wp, nbytes)
    return out


def attention_status(device="cuda") -> int:
    """Status word of the attention kernels on a device (0 = ok, 5 = a device-side
    wait gave up since the last reading); synchronises."""
    with torch.cuda.device(device):
        return int(_sls.lib().sls_attention_status(
            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))
