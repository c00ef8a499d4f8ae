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
import math
from typing import Optional

import torch

import paper_2607_19368_gb300 as _sls

__all__ = ["SLS_F16", "Rope", "qkv_append", "attention_prefill", "attention_decode",
           "attention_status"]

SLS_F16 = 2

_vp, _i64, _i32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float,
                              ctypes.c_size_t)


class _Cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("dtype", _i32), ("kv_heads", _i32), ("head_dim", _i32),
                ("page_size", _i32), ("num_pages", _i64), ("page_stride", _i64),
                ("slot_stride", _i64), ("head_stride", _i64), ("page_table", _vp),
                ("table_ld", _i64), ("max_pages", _i32), ("kv_lens", _vp), ("batch", _i64)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class _Rope(ctypes.Structure):
    _fields_ = [("inv_freq", _vp), ("pairs", _i32), ("interleaved", _i32), ("scale", _f32)]


_P = ctypes.POINTER

# name -> (restype, argtypes); the attention part of include/sls.h
EXPORTED = {
    "sls_qkv_append": (_i32, [_P(_Rows), _P(_Rows), _P(_Rows), _i64, _i32, _P(_Cache), _vp, _vp,
                              _vp, _vp, _f32, _P(_Rope), _P(_Rows), _vp]),
    "sls_attention_prefill_workspace_size": (_sz, [_i64, _i32, _P(_Cache)]),
    "sls_attention_prefill": (_i32, [_P(_Rows), _i64, _i32, _P(_Cache), _vp, _i32, _f32,
                                     _P(_Rows), _vp, _sz, _vp]),
    "sls_attention_decode_workspace_size": (_sz, [_i32, _P(_Cache)]),
    "sls_attention_decode": (_i32, [_P(_Rows), _i32, _P(_Cache), _f32, _P(_Rows), _vp, _sz,
                                    _vp]),
    "sls_attention_status": (_i32, [_vp]),
}

_CODES = {torch.bfloat16: 1, torch.float16: SLS_F16}


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
        self._c = _Rope(self.inv_freq.data_ptr(), self.inv_freq.numel(), int(self.interleaved),
                        self.scale)

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


def _code(t: torch.Tensor) -> int:
    c = _CODES.get(t.dtype)
    if c is None:
        raise TypeError(f"unsupported attention dtype {t.dtype} (bfloat16 or float16)")
    return c


def _rows(name: str, t: torch.Tensor, dtype, head_dim: int) -> _Rows:
    if t.dim() != 3 or t.shape[2] != head_dim or t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{name}: tokens x heads x {head_dim} of {dtype} on the GPU")
    st, sh, se = t.stride()
    if se != 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    # the stride of a dimension of one entry says nothing
    if t.shape[1] == 1:
        sh = head_dim
    if t.shape[0] <= 1:
        st = sh * t.shape[1]
    return _Rows(t.data_ptr(), st, sh)


def _ints(name: str, t: torch.Tensor, n: Optional[int] = None) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous() \
            or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name}: a contiguous int32 CUDA tensor"
                         + (f" of {n} entries" if n is not None else ""))
    return t


def _cache(cache_k, cache_v, page_table, kv_lens) -> _Cache:
    code = _code(cache_k)
    if cache_k.dim() != 4 or cache_v.shape != cache_k.shape or cache_v.dtype != cache_k.dtype \
            or not cache_k.is_cuda or not cache_v.is_cuda:
        raise ValueError("cache_k, cache_v: pages x page_size x kv_heads x head_dim, alike, on "
                         "the GPU")
    sp, ss, sh, se = cache_k.stride()
    if se != 1 or cache_v.stride() != cache_k.stride():
        raise ValueError("cache_k, cache_v: equal strides, contiguous heads")
    _ints("kv_lens", kv_lens)
    B = kv_lens.shape[0]
    if page_table.dim() != 2 or page_table.shape[0] != B or page_table.dtype != torch.int32 \
            or not page_table.is_cuda or page_table.stride(1) != 1:
        raise ValueError("page_table: B x max_pages int32 on the GPU, contiguous rows")
    n, ps, H, hd = cache_k.shape
    if H == 1:
        sh = hd
    if n <= 1:
        sp = ps * max(ss, sh * H)
    cols = page_table.shape[1]
    return _Cache(cache_k.data_ptr(), cache_v.data_ptr(), code, H, hd, ps, n, sp, ss, sh,
                  page_table.data_ptr(), max(page_table.stride(0), cols), cols,
                  kv_lens.data_ptr(), B)


def _weight(name: str, w: Optional[torch.Tensor], dtype, head_dim: int):
    if w is None:
        return None
    if w.dtype != dtype or w.shape != (head_dim,) or not w.is_contiguous() or not w.is_cuda:
        raise ValueError(f"{name}: {head_dim} contiguous elements of {dtype} on the GPU")
    return w.data_ptr()


def _done(fn: str, st: int, t: torch.Tensor):
    _sls._check(fn, st)
    if _sls._CHECK_STATUS:
        with torch.cuda.device(t.device):
            st = int(_sls.lib().sls_attention_status(_sls._stream(t)))
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
    c = _cache(cache_k, cache_v, page_table, kv_lens)
    dt, hd = cache_k.dtype, cache_k.shape[3]
    T, Hq = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty((T, Hq, hd), dtype=q.dtype, device=q.device)
    rq, rk, rv, ro = (_rows("q", q, dt, hd), _rows("k", k, dt, hd), _rows("v", v, dt, hd),
                      _rows("out", out, dt, hd))
    want = (T, c.kv_heads, hd)
    if tuple(k.shape) != want or tuple(v.shape) != want or out.shape != q.shape:
        raise ValueError("k and v: one row per token of q and key head; out: the shape of q")
    if cu_seqlens is not None:
        _ints("cu_seqlens", cu_seqlens, c.batch + 1)
    elif T != c.batch:
        raise ValueError("without cu_seqlens q has one token per sequence")
    if positions is not None:
        _ints("positions", positions, T)
    st = _sls.lib().sls_qkv_append(
        rq, rk, rv, T, Hq, c, None if cu_seqlens is None else cu_seqlens.data_ptr(),
        None if positions is None else positions.data_ptr(),
        _weight("q_weight", q_weight, dt, hd), _weight("k_weight", k_weight, dt, hd), eps,
        None if rope is None else rope._c, ro, _sls._stream(q))
    _done("sls_qkv_append", st, q)
    return out


def _attention_args(q, cache_k, out, scale):
    dt, hd = cache_k.dtype, cache_k.shape[3]
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out: the shape of q")
    return (_rows("q", q, dt, hd), _rows("out", out, dt, hd), out,
            1.0 / math.sqrt(hd) if scale is None else float(scale))


def _scratch(nbytes: int, workspace: Optional[torch.Tensor], device):
    """(pointer, bytes, tensor) of a caller's workspace (a uint8 tensor) or of one
    for this call."""
    if workspace is None:
        if nbytes == 0:
            return None, 0, None
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    elif not workspace.is_cuda or workspace.dtype != torch.uint8:
        raise ValueError("workspace: a uint8 CUDA tensor")
    return workspace.data_ptr(), workspace.numel(), workspace


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
    c = _cache(cache_k, cache_v, page_table, kv_lens)
    rq, ro, out, scale = _attention_args(q, cache_k, out, scale)
    _ints("cu_seqlens", cu_seqlens, c.batch + 1)
    T, Hq = q.shape[0], q.shape[1]
    L = _sls.lib()
    wp, wn, keep = _scratch(L.sls_attention_prefill_workspace_size(T, Hq, c), workspace, q.device)
    st = L.sls_attention_prefill(rq, T, Hq, c, cu_seqlens.data_ptr(), int(causal), scale, ro, wp,
                                 wn, _sls._stream(q))
    _done("sls_attention_prefill", st, q)
    return out


def attention_decode(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                     page_table: torch.Tensor, kv_lens: torch.Tensor,
                     scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One token per sequence (q: B x q_heads x head_dim) over all kv_lens tokens of
    its sequence.  Returns q's shape; a sequence of length 0 gives zeros."""
    c = _cache(cache_k, cache_v, page_table, kv_lens)
    rq, ro, out, scale = _attention_args(q, cache_k, out, scale)
    if q.shape[0] != c.batch:
        raise ValueError("q: one token per sequence")
    Hq = q.shape[1]
    L = _sls.lib()
    wp, wn, keep = _scratch(L.sls_attention_decode_workspace_size(Hq, c), workspace, q.device)
    st = L.sls_attention_decode(rq, Hq, c, scale, ro, wp, wn, _sls._stream(q))
    _done("sls_attention_decode", st, q)
    return out


def attention_status(device="cuda") -> int:
    """Status word of the attention kernels on a device (0 = ok, 5 = a device-side
    wait gave up since the last reading); synchronises."""
    with torch.cuda.device(device):
        return int(_sls.lib().sls_attention_status(
            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))
