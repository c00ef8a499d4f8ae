"""Refusals of the attention calls and the frequencies of the rotation, without a GPU."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def sls():
    from paper_2607_19368_gb300 import build
    build.build()
    import paper_2607_19368_gb300 as sls
    return sls


class _Cache(ctypes.Structure):
    """sls_kv_cache_t as the header declares it."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("page_size", ctypes.c_int), ("num_pages", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("page_table", ctypes.c_void_p),
                ("table_ld", ctypes.c_int64), ("max_pages", ctypes.c_int),
                ("kv_lens", ctypes.c_void_p), ("batch", ctypes.c_int64)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _Rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("pairs", ctypes.c_int),
                ("interleaved", ctypes.c_int), ("scale", ctypes.c_float)]


def test_packed_layouts_are_the_structures(sls):
    from paper_2607_19368_gb300 import attention as A
    for packed, kind in ((A._CACHE, _Cache), (A._ROWS, _Rows), (A._ROPE, _Rope)):
        # one odd value per field, in the header's order
        vals = [float(i + 1) if f[1] is ctypes.c_float else 1001 + i
                for i, f in enumerate(kind._fields_)]
        assert packed.pack(*vals).ljust(ctypes.sizeof(kind), b"\0") == bytes(kind(*vals))


def cache(sls, **kw):
    a = dict(k=256, v=256, dtype=1, kv_heads=2, head_dim=64, page_size=16, num_pages=4,
             page_stride=16 * 128, slot_stride=128, head_stride=64, page_table=256, table_ld=2,
             max_pages=2, kv_lens=256, batch=2)
    a.update(kw)
    return ctypes.byref(_Cache(**a))


def rows(data=256, token=512, head=64):
    return ctypes.byref(_Rows(data, token, head))


BAD_CACHE = [
    (dict(dtype=0), 2), (dict(dtype=3), 2), (dict(head_dim=132), 2), (dict(head_dim=60), 2),
    (dict(head_dim=0), 2), (dict(page_size=8), 2), (dict(page_size=48), 2),
    (dict(page_size=2048), 2), (dict(kv_heads=3), 1), (dict(kv_heads=0), 1),
    (dict(slot_stride=60), 1), (dict(slot_stride=132), 1), (dict(head_stride=4), 1),
    (dict(page_stride=-8), 1), (dict(table_ld=1), 1), (dict(k=8), 1), (dict(v=0), 1),
    (dict(kv_lens=0), 1), (dict(page_table=0), 1), (dict(batch=-1), 1), (dict(max_pages=-1), 1),
    (dict(num_pages=1 << 40), 2), (dict(kv_heads=1, q_heads=129), 2),
]


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_caches_that_are_refused(sls, change, status):
    L = sls.lib()
    change = dict(change)
    Hq = change.pop("q_heads", 4)
    c = cache(sls, **change)
    r = rows()
    assert L.sls_attention_decode(r, Hq, c, 1.0, r, None, 0, None) == status
    assert L.sls_attention_prefill(r, 3, Hq, c, 256, 1, 1.0, r, None, 0, None) == status
    assert L.sls_qkv_append(r, r, r, 3, Hq, c, 256, None, None, None, 1e-6, None, r,
                            None) == status


def test_rows_and_options_that_are_refused(sls):
    L, c, r = sls.lib(), cache(sls), rows()

    def rope(inv_freq, pairs):
        return ctypes.byref(_Rope(inv_freq, pairs, 0, 1.0))

    def append(q=r, k=r, v=r, T=3, cu=256, qw=None, eps=1e-6, rope=None, out=r, Hq=4):
        return L.sls_qkv_append(q, k, v, T, Hq, c, cu, None, qw, None, eps, rope, out, None)

    for bad in (rows(data=8), rows(data=0), rows(token=4), rows(head=4), rows(head=32),
                rows(token=-512), None):
        assert append(q=bad) == 1 and append(k=bad) == 1 and append(v=bad) == 1
        assert append(out=bad) == 1
        assert L.sls_attention_prefill(bad, 3, 4, c, 256, 1, 1.0, r, None, 0, None) == 1
        assert L.sls_attention_decode(r, 4, c, 1.0, bad, None, 0, None) == 1
    assert append(T=-1) == 1 and append(T=3, cu=None) == 1 and append(qw=8) == 1
    assert append(eps=-1.0) == 1 and append(eps=math.nan) == 1 and append(Hq=3) == 1
    assert append(Hq=0) == 1
    assert append(rope=rope(256, 33)) == 1 and append(rope=rope(None, 8)) == 1
    assert append(rope=rope(256, -1)) == 1
    assert L.sls_attention_prefill(r, 3, 4, c, None, 1, 1.0, r, None, 0, None) == 1
    assert L.sls_attention_prefill(r, 3, 4, None, 256, 1, 1.0, r, None, 0, None) == 1
    # nothing to do is no error
    assert L.sls_attention_prefill(r, 0, 4, c, 256, 1, 1.0, r, None, 0, None) == 0
    assert append(T=0) == 0
    assert L.sls_attention_decode(r, 4, cache(sls, batch=0), 1.0, r, None, 0, None) == 0


def test_binding_refuses_what_it_cannot_pass(sls):
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 2, dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        sls.attention_decode(q, k, k, t, n)                       # not on the GPU
    with pytest.raises(TypeError):
        sls.attention_decode(q.float(), k.float(), k.float(), t, n)
    with pytest.raises(ValueError):
        sls.Rope(torch.zeros(8))
    with pytest.raises(ValueError):
        sls.Rope.make(7)
    with pytest.raises(ValueError):
        sls.Rope.make(8, factor=0.5)


def test_frequencies(sls, monkeypatch):
    """base^(-2i/rot); all divided by the factor; with a length, fast ones kept,
    slow ones divided, a blend between that is linear in the number of turns."""
    seen = []
    monkeypatch.setattr(sls.Rope, "__init__",
                        lambda self, f, interleaved=False, scale=1.0: seen.append(f))
    sls.Rope.make(64, base=500.0, device="cpu")
    sls.Rope.make(64, base=500.0, factor=4.0, device="cpu")
    sls.Rope.make(64, base=500.0, factor=4.0, original_length=1000, slow_turns=2.0,
                  fast_turns=20.0, device="cpu")
    for i in range(32):
        f = 500.0 ** (-i / 32)
        turns = 1000 * f / (2 * math.pi)
        part = min(1.0, max(0.0, (turns - 2.0) / 18.0))
        assert abs(seen[0][i].item() - f) <= 2 ** -24 * f
        assert abs(seen[1][i].item() - f / 4) <= 2 ** -24 * f
        assert abs(seen[2][i].item() - (part * f + (1 - part) * f / 4)) <= 2 ** -23 * f
    assert ctypes.sizeof(ctypes.c_void_p) == 8
