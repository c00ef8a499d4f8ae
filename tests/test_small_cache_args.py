"""Refusals of the calls that make the cache smaller, without a GPU."""
import ctypes
import math
import weakref

import pytest
import torch

from tests.test_attention_args import _Cache, _Rope, _Rows, rows


@pytest.fixture(scope="module")
def sls():
    from paper_2607_19368_gb300 import build
    build.build()
    import paper_2607_19368_gb300 as sls
    return sls


class _Scales(ctypes.Structure):
    """sls_kv_scales_t as the header declares it."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("block", ctypes.c_int),
                ("page_stride", ctypes.c_int64), ("block_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _Weights(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


def test_packed_layouts_are_the_structures(sls):
    from paper_2607_19368_gb300 import small_cache as C
    for packed, kind in ((C._SCALES, _Scales), (C._WEIGHTS, _Weights)):
        vals = [1001 + i for i, _ in enumerate(kind._fields_)]
        assert packed.pack(*vals).ljust(ctypes.sizeof(kind), b"\0") == bytes(kind(*vals))


def cache(**kw):
    a = dict(k=256, v=256, dtype=3, kv_heads=2, head_dim=64, page_size=32, num_pages=4,
             page_stride=32 * 128, slot_stride=128, head_stride=64, page_table=256, table_ld=2,
             max_pages=2, kv_lens=256, batch=2)
    a.update(kw)
    return ctypes.byref(_Cache(**a))


def scales(**kw):
    a = dict(k=256, v=256, block=16, page_stride=4, block_stride=2, head_stride=1)
    a.update(kw)
    return ctypes.byref(_Scales(**a))


def weights(**kw):
    a = dict(data=256, page_stride=64, head_stride=32)
    a.update(kw)
    return ctypes.byref(_Weights(**a))


def calls(L, c, s, dtype=1, Hq=4, T=3, evict=True):
    """Every call of the family: name -> status.  All are refused, the last resort being a
    workspace that is missing; eviction, which needs none, is left out where it would run."""
    r, w = rows(), weights()
    got = {
        "append": L.sls_qkv_append_q8(r, r, r, T, Hq, c, s, dtype, 256, None, None, None, 1e-6,
                                      None, r, None),
        "prefill": L.sls_attention_prefill_q8(r, T, Hq, c, s, dtype, 256, 1, 1.0, r, None, 0, None),
        "decode": L.sls_attention_decode_q8(r, Hq, c, s, dtype, 1.0, r, None, 0, None),
        "weights": L.sls_attention_weights(r, T, Hq, c, s, dtype, 256, 1, 1.0, w, None, 0, None),
    }
    if evict:
        got["evict"] = L.sls_cache_evict(c, s, w, 8, 1, 2, 256, 256, None)
    return got


BAD_CACHE = [
    (dict(dtype=1), 2), (dict(dtype=5), 2), (dict(head_dim=136), 2), (dict(head_dim=72), 2),
    (dict(head_dim=0), 2), (dict(page_size=8), 2), (dict(page_size=48), 2),
    (dict(kv_heads=0), 1), (dict(slot_stride=60), 1), (dict(slot_stride=136), 1),
    (dict(head_stride=8), 1), (dict(page_stride=-16), 1), (dict(table_ld=1), 1), (dict(k=8), 1),
    (dict(kv_lens=0), 1), (dict(page_table=0), 1), (dict(batch=-1), 1), (dict(max_pages=-1), 1),
    (dict(num_pages=1 << 40), 2), (dict(num_pages=0), 1),
]


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_caches_that_are_refused(sls, change, status):
    assert set(calls(sls.lib(), cache(**change), scales()).values()) == {status}


BAD_SCALES = [(dict(k=0), 1), (dict(k=2), 1), (dict(block=8), 2), (dict(block=24), 2),
              (dict(block=64), 2), (dict(block=256), 2), (dict(page_stride=0), 1),
              (dict(block_stride=-1), 1), (dict(head_stride=0), 1)]


@pytest.mark.parametrize("change,status", BAD_SCALES)
def test_scales_that_are_refused(sls, change, status):
    assert set(calls(sls.lib(), cache(), scales(**change)).values()) == {status}


def test_values_and_their_scales_are_wanted_where_they_are_read(sls):
    L = sls.lib()
    for c, s in ((cache(v=0), scales()), (cache(), scales(v=0))):
        got = calls(L, c, s)
        # the weights read keys alone; what stops them here is the missing workspace, or GPU
        assert got.pop("weights") in (3, 4) and set(got.values()) == {1}
    # a cache of codes without scales, and scales with a 16-bit cache
    got = calls(L, cache(), None)
    assert got.pop("weights") == 2 and got.pop("evict") == 2 and set(got.values()) == {1}
    assert set(calls(L, cache(dtype=1), scales()).values()) == {2}


def test_options_that_are_refused(sls):
    L, c, s, r = sls.lib(), cache(), scales(), rows()

    def rope(inv_freq, pairs):
        return ctypes.byref(_Rope(inv_freq, pairs, 0, 1.0))

    def append(q=r, k=r, v=r, T=3, cu=256, qw=None, eps=1e-6, rope=None, out=r, Hq=4, dtype=1):
        return L.sls_qkv_append_q8(q, k, v, T, Hq, c, s, dtype, cu, None, qw, None, eps, rope,
                                   out, None)

    for bad in (rows(data=8), rows(data=0), rows(token=4), rows(head=4), rows(head=32),
                rows(token=-512), None):
        assert append(q=bad) == 1 and append(k=bad) == 1 and append(v=bad) == 1
        assert append(out=bad) == 1
        assert L.sls_attention_prefill_q8(bad, 3, 4, c, s, 1, 256, 1, 1.0, r, None, 0, None) == 1
        assert L.sls_attention_decode_q8(r, 4, c, s, 1, 1.0, bad, None, 0, None) == 1
        assert L.sls_attention_weights(bad, 3, 4, c, s, 1, 256, 1, 1.0, weights(), None, 0,
                                       None) == 1
    assert append(T=-1) == 1 and append(T=3, cu=None) == 1 and append(qw=8) == 1
    assert append(eps=-1.0) == 1 and append(eps=math.nan) == 1 and append(Hq=3) == 1
    assert append(dtype=3) == 2 and append(Hq=0) == 1
    assert append(rope=rope(256, 33)) == 1 and append(rope=rope(None, 8)) == 1
    assert append(T=0) == 0
    for dtype in (0, 3, 4):
        assert set(calls(L, c, s, dtype=dtype, evict=False).values()) == {2}
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert L.sls_attention_decode_q8(r, 4, c, s, 1, scale, r, None, 0, None) == 1
        assert L.sls_attention_prefill_q8(r, 3, 4, c, s, 1, 256, 1, scale, r, None, 0, None) == 1
        assert L.sls_attention_weights(r, 3, 4, c, s, 1, 256, 1, scale, weights(), None, 0,
                                       None) == 1
    # offsets, workspaces
    assert L.sls_attention_prefill_q8(r, 3, 4, c, s, 1, None, 1, 1.0, r, None, 0, None) == 1
    assert L.sls_attention_weights(r, 3, 4, c, s, 1, None, 1, 1.0, weights(), None, 0, None) == 1
    assert L.sls_attention_prefill_q8(r, 3, 4, c, s, 1, 256, 1, 1.0, r, 256, 16, None) == 3
    # 16-bit keys of another type than the queries'
    wide = cache(dtype=2)
    assert L.sls_attention_weights(r, 3, 4, wide, None, 1, 256, 1, 1.0, weights(), None, 0,
                                   None) == 2
    for bad in (None, weights(data=0), weights(data=8), weights(page_stride=-4),
                weights(page_stride=62), weights(page_stride=0), weights(head_stride=30),
                weights(head_stride=28)):
        assert L.sls_attention_weights(r, 3, 4, c, s, 1, 256, 1, 1.0, bad, None, 0, None) == 1
        assert L.sls_cache_evict(c, s, bad, 8, 1, 2, 256, 256, None) == 1

    def evict(keep=8, first=1, last=2, kept=256, lens=256):
        return L.sls_cache_evict(c, s, weights(), keep, first, last, kept, lens, None)

    assert evict(keep=-1) == 1 and evict(first=-1) == 1 and evict(last=-1) == 1
    assert evict(first=4, last=5) == 1 and evict(kept=None) == 1 and evict(lens=None) == 1
    assert evict(lens=512) == 1 and evict(keep=1 << 40) == 1
    # sums past 64 bits
    assert evict(first=(1 << 63) - 1, last=1) == 1 and evict(first=1, last=(1 << 63) - 1) == 1
    # more sequences than a packed call looks through
    many = cache(batch=65537)
    got = calls(L, many, s, evict=False)
    assert got["append"] == got["prefill"] == got["weights"] == 2


def test_nothing_to_do_is_no_error(sls):
    L, r = sls.lib(), rows()
    none, s = cache(batch=0), scales()
    assert L.sls_attention_decode_q8(r, 4, none, s, 1, 1.0, r, None, 0, None) == 0
    assert L.sls_attention_prefill_q8(r, 0, 4, none, s, 1, 256, 1, 1.0, r, None, 0, None) == 0
    assert L.sls_qkv_append_q8(r, r, r, 0, 4, none, s, 1, None, None, None, None, 1e-6, None, r,
                               None) == 0
    assert L.sls_attention_weights(r, 0, 4, none, s, 1, None, 1, 1.0, weights(), None, 0, None) == 0
    assert L.sls_cache_evict(none, s, weights(), 8, 1, 2, None, None, None) == 0


def test_binding_refuses_what_it_cannot_pass(sls):
    k = torch.zeros(4, 32, 2, 64, dtype=torch.int8)
    f = torch.zeros(4, 2, 2)
    t = torch.zeros(2, 2, dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    w = torch.zeros(4, 2, 32)
    with pytest.raises(ValueError):
        sls.attention_decode_q8(q, k, k, f, f, t, n)                   # not on the GPU
    with pytest.raises(TypeError):
        sls.attention_decode_q8(q, k.bfloat16(), k.bfloat16(), f, f, t, n)
    with pytest.raises(TypeError):
        sls.attention_decode_q8(q.float(), k, k, f, f, t, n)
    with pytest.raises(TypeError):
        sls.attention_prefill_q8(q.int(), k, k, f, f, t, n, n)
    with pytest.raises(TypeError):
        sls.qkv_append_q8(q, q, q, q, q, f, f, t, n)
    with pytest.raises(TypeError):
        sls.attention_weights(q, k, t, n, w)                           # codes without scales
    with pytest.raises(TypeError):
        sls.cache_evict(k, k, t, n, w, 4)
    with pytest.raises(TypeError):
        sls.attention_decode(q, k, k, t, n)                            # the 16-bit call


def test_arguments_live_until_the_call(sls, monkeypatch):
    """Tensors that a caller makes for one call are not freed before its workspace is allocated,
    which could take their memory, nor before its launches."""
    from paper_2607_19368_gb300 import small_cache as C
    refs, alive = [], []

    def temp(*shape, dtype=torch.int32):
        t = torch.zeros(*shape, dtype=dtype)
        refs.append(weakref.ref(t))
        return t

    def look(*a, **kw):
        alive.append([r() is not None for r in refs])
        return torch.empty(16, dtype=torch.uint8)

    k = torch.zeros(4, 32, 2, 64, dtype=torch.int8)
    monkeypatch.setattr(C, "_cache", lambda *a: (b"", k.shape, k.dtype, 0, 2, 2))
    for name in ("_rows", "_ints", "_weight", "_weights"):
        monkeypatch.setattr(C, name, lambda *a: 256)
    monkeypatch.setattr(C, "_scales", lambda *a: (b"", 16))
    monkeypatch.setattr(C, "_bytes", lambda *a: 16)
    monkeypatch.setattr(C, "_attention_rows", lambda q, out, *a: (b"", b"", q, 1.0))
    monkeypatch.setattr(C, "_scratch", look)
    monkeypatch.setattr(C, "_call", look)
    f32, bf16 = torch.float32, torch.bfloat16
    q = torch.zeros(2, 4, 64, dtype=bf16)
    C.attention_weights(temp(2, 4, 64, dtype=bf16), k, temp(2, 2), temp(2),
                        temp(4, 2, 32, dtype=f32), temp(3), k_scale=temp(4, 2, 2, dtype=f32))
    assert alive == [[True] * 6] * 2
    refs.clear(), alive.clear()
    C.attention_prefill_q8(temp(2, 4, 64, dtype=bf16), k, k, temp(4, 2, 2, dtype=f32),
                           temp(4, 2, 2, dtype=f32), temp(2, 2), temp(2), temp(3), out=q)
    assert alive == [[True] * 6] * 2
    refs.clear(), alive.clear()
    C.attention_decode_q8(temp(2, 4, 64, dtype=bf16), k, k, temp(4, 2, 2, dtype=f32),
                          temp(4, 2, 2, dtype=f32), temp(2, 2), temp(2), out=q)
    assert alive == [[True] * 5] * 2
    refs.clear(), alive.clear()
    C.qkv_append_q8(q, temp(2, 2, 64, dtype=bf16), temp(2, 2, 64, dtype=bf16), k, k,
                    temp(4, 2, 2, dtype=f32), temp(4, 2, 2, dtype=f32), temp(2, 2), temp(2),
                    temp(3), temp(2), temp(64, dtype=bf16), temp(64, dtype=bf16))
    assert alive == [[True] * 10]
