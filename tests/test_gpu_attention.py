"""The attention calls against a float64 statement of their definitions
(tests/attention_ref.py): append with norm and rotation, packed prefill, decode
over the paged cache, at lengths, head layouts, page sizes, strides and masks
where a tiled kernel can go wrong.  Slots that no sequence covers hold NaN in
every case, so nothing but the covered ones may reach a result."""
import math

import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def prefill(sls, b, **kw):
    return sls.attention_prefill(b["q"], b["k"], b["v"], b["table"], b["kv_lens"], b["cu"], **kw)


def decode(sls, b, **kw):
    return sls.attention_decode(b["q"], b["k"], b["v"], b["table"], b["kv_lens"], **kw)


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

APPEND = [
    # new, m, Hq, Hkv, hd, page, pairs, interleaved, norm, positions
    ([1], [1], 4, 1, 128, 16, 64, False, True, True),
    ([1, 1, 1], [5, 700, 33], 28, 4, 128, 64, 64, False, True, True),
    ([5, 0, 17, 130], [5, 9, 40, 1000], 14, 2, 64, 16, 32, True, True, True),
    ([33, 8], [40, 8], 6, 3, 96, 32, 48, False, False, True),
    ([33, 8], [40, 8], 6, 3, 96, 32, 12, False, True, True),      # halves of 12: no whole vectors
    ([20, 7], [50, 7], 10, 2, 80, 16, 10, False, True, False),    # halves of 10, cache positions
    ([20, 7], [50, 7], 10, 2, 80, 16, 9, True, True, True),       # an odd number of pairs
    ([9], [4], 4, 4, 8, 16, 4, False, True, True),                # more tokens than cache places
    ([64], [64], 8, 8, 40, 1024, 0, False, True, True),           # no rotation
    ([300], [4000], 40, 8, 128, 128, 64, True, False, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", APPEND)
def test_append(sls, case, dtype):
    new, m, Hq, Hkv, hd, page, pairs, inter, norm, use_pos = case
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=len(str(case)))
    T = sum(new)
    g = torch.Generator("cuda").manual_seed(3)
    qkv = torch.randn(T, Hq + 2 * Hkv, hd, generator=g, device="cuda").to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    qw = kw = None
    if norm:
        qw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
        kw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
    pos = torch.randint(0, 131072, (T,), generator=g, device="cuda", dtype=torch.int32)
    pos = pos if use_pos else None
    f = sls.Rope.make(max(2, 2 * pairs), base=1e6).inv_freq[:pairs].contiguous()
    rope = sls.Rope(f, interleaved=inter, scale=1.25) if pairs else None
    qo, K, V, qb, bK = R.append(q, k, v, b, pos, qw, kw, 1e-5, f if pairs else None, inter, 1.25)
    got = sls.qkv_append(q, k, v, b["k"], b["v"], b["table"], b["kv_lens"], cu_seqlens=b["cu"],
                         positions=pos, q_weight=qw, k_weight=kw, eps=1e-5, rope=rope)
    R.check(got, qo, qb, "q")
    hole = torch.isnan(K)
    assert torch.equal(torch.isnan(b["k"]), hole) and torch.equal(torch.isnan(b["v"]), hole)
    R.check(b["k"].double().masked_fill(hole, 0), K.masked_fill(hole, 0),
            bK.masked_fill(hole, 0), "k")
    assert torch.equal(b["v"].double().masked_fill(hole, 0), V.masked_fill(hole, 0))
    # in place, and one token per sequence without offsets
    again = sls.qkv_append(q, k, v, b["k"], b["v"], b["table"], b["kv_lens"], cu_seqlens=b["cu"],
                           positions=pos, q_weight=qw, k_weight=kw, eps=1e-5, rope=rope, out=q)
    assert again.data_ptr() == q.data_ptr() and torch.equal(again, got)
    if all(n == 1 for n in new):
        q2 = qkv[:, :Hq].clone()
        one = sls.qkv_append(got, k, v, b["k"], b["v"], b["table"], b["kv_lens"], positions=pos,
                             k_weight=kw, eps=1e-5, rope=rope, out=q2)
        assert one is q2


def test_append_far_positions(sls):
    """Angles at positions up to 2^22 come from the exact product of position and
    frequency."""
    hd, T = 128, 64
    b = R.make_batch([T], [T], 2, 1, hd, 64, torch.float16, seed=5)
    g = torch.Generator("cuda").manual_seed(6)
    x = torch.randn(T, 4, hd, generator=g, device="cuda").half()
    pos = torch.randint(1 << 21, 1 << 22, (T,), generator=g, device="cuda", dtype=torch.int32)
    rope = sls.Rope.make(hd, base=10000.0)
    qo, K, V, qb, bK = R.append(x[:, :2], x[:, 2:3], x[:, 3:], b, pos, None, None, 0.0,
                                rope.inv_freq, False, 1.0)
    got = sls.qkv_append(x[:, :2], x[:, 2:3], x[:, 3:], b["k"], b["v"], b["table"], b["kv_lens"],
                         cu_seqlens=b["cu"], positions=pos, rope=rope)
    R.check(got, qo, qb, "q")


def test_append_skips_what_has_no_place(sls):
    """Tokens past the last sequence, page numbers outside the cache and indices
    past the table: nothing is written, the queries are."""
    b = R.make_batch([4, 4], [20, 300], 4, 2, 64, 16, torch.bfloat16, seed=7)
    cols = b["table"].shape[1]
    b["kv_lens"][1] = cols * 16 + 2        # the last two new tokens lie past the table
    b["table"][0, 1] = -5                  # sequence 0's second page is none
    b["table"][1, cols - 1] = 1 << 30
    x = torch.randn(11, 8, 64, device="cuda").bfloat16()
    before = b["k"].clone(), b["v"].clone()
    out = sls.qkv_append(x[:, :4], x[:, 4:6], x[:, 6:], b["k"], b["v"], b["table"], b["kv_lens"],
                         cu_seqlens=b["cu"])
    assert torch.equal(out, x[:, :4])
    for a, c in zip(before, (b["k"], b["v"])):
        assert torch.equal(a.view(torch.int16), c.view(torch.int16))


# ---------------------------------------------------------------------------
# prefill
# ---------------------------------------------------------------------------

PREFILL = [
    # new, m, Hq, Hkv, hd, page, causal
    ([1], [1], 1, 1, 64, 16, True),
    ([1], [1], 28, 4, 128, 64, True),
    ([2], [130], 8, 8, 128, 64, True),
    ([17], [17], 28, 4, 128, 64, True),
    ([128], [128], 8, 8, 128, 128, True),
    ([129], [129], 4, 4, 128, 128, True),
    ([255, 257, 256], [255, 257, 256], 4, 2, 128, 16, True),
    ([300], [300], 28, 4, 128, 64, True),
    ([300, 1, 0, 77], [300, 500, 30, 77], 14, 2, 64, 32, True),
    ([137], [137], 28, 4, 128, 64, True),
    ([50, 50], [50, 1333], 32, 8, 128, 16, False),
    ([64, 10], [20, 0], 4, 2, 64, 16, True),             # rows before the first key; no keys
    ([64, 10], [20, 0], 4, 2, 64, 16, False),
    ([0, 0], [5, 0], 4, 2, 64, 16, True),                # no rows at all
    ([700], [2100], 10, 2, 80, 32, True),
    ([333], [333], 9, 3, 96, 16, True),
    ([65], [400], 40, 40, 8, 16, True),
    ([200], [200], 128, 1, 64, 64, True),                # a head group that fills a tile
    ([90], [90], 66, 1, 32, 64, True),                   # a group that leaves half a tile
    ([400, 3], [400, 2000], 25, 5, 72, 256, True),
    ([40, 41, 42, 43, 44, 45, 46, 47] * 5, [40, 41, 42, 43, 44, 45, 46, 999] * 5, 8, 2, 64, 16,
     True),
    ([1024], [1024], 16, 2, 128, 1024, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", PREFILL)
def test_prefill(sls, case, dtype):
    new, m, Hq, Hkv, hd, page, causal = case
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=len(str(case)))
    want, bound = R.attention(b, causal)
    R.check(prefill(sls, b, causal=causal), want, bound, str(case))


@pytest.mark.parametrize("order", ["tokens", "heads"])
def test_prefill_strides(sls, order):
    """A cache with heads outside slots, queries that are slices of a projection,
    an output with gaps, another scale, another stream."""
    b = R.make_batch([150, 61], [150, 300], 8, 2, 128, 32, torch.bfloat16, seed=11, order=order)
    T = 211
    wide = torch.zeros(T, 8 + 5, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:11] = b["q"]
    b["q"] = wide[:, 3:11]
    room = torch.full((T, 10, 136), 3.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, 1:9, :128]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = prefill(sls, b, scale=0.05, out=out)
    side.synchronize()
    assert got.data_ptr() == out.data_ptr()
    want, bound = R.attention(b, True, 0.05)
    R.check(out, want, bound)
    keep = torch.ones_like(room, dtype=torch.bool)
    keep[:, 1:9, :128] = False
    assert (room[keep] == 3.0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k", "v"])
def test_prefill_later_token_does_not_reach_earlier_rows(sls, where, bad):
    """A NaN or infinity in a token's key or value changes no row that does not
    see the token, in its own tile either."""
    b = R.make_batch([200], [290], 4, 2, 64, 16, torch.bfloat16, seed=13)
    want, bound = R.attention(b)
    x = 230                                       # cache index of the token: row 140 on sees it
    b[where][b["table"][0, x // 16].long(), x % 16, :, 5] = bad
    got = prefill(sls, b)
    R.check(got[:140], want[:140], bound[:140])
    ref, _ = R.attention(b)
    assert torch.equal(torch.isnan(got[140:]), torch.isnan(ref[140:]))
    assert torch.equal(torch.isinf(got[140:]), torch.isinf(ref[140:]))


def test_prefill_large_and_low_scores(sls):
    """Scores of +-thousands: the weights fall on one key or a few, none overflows."""
    b = R.make_batch([130], [130], 4, 4, 64, 64, torch.bfloat16, seed=17, q_scale=300.0)
    want, bound = R.attention(b)
    got = prefill(sls, b)
    R.check(got, want, bound)
    lo = torch.finfo(torch.bfloat16).min / 8
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    b["k"][..., 0] = lo                             # every score about the type's lowest value
    want, bound = R.attention(b)
    R.check(prefill(sls, b), want, bound)


CUT = [
    # few rows against many cached tokens: items fall to several CTAs
    ([1], [3000], 28, 4, 128, 64, True),
    ([50], [10050], 28, 4, 128, 64, True),
    ([3, 0, 200, 1], [2500, 40, 2300, 6000], 8, 2, 128, 16, True),
    ([20, 5, 9], [4100, 0, 3], 6, 3, 96, 32, True),          # sequences without keys, rows before them
    ([64], [5000], 10, 2, 64, 128, False),
    ([100, 30], [7000, 2049], 24, 8, 40, 1024, True),
    ([7], [2047], 66, 1, 128, 16, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CUT)
def test_prefill_cut(sls, case, dtype):
    new, m, Hq, Hkv, hd, page, causal = case
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=61)
    want, bound = R.attention(b, causal)
    got = prefill(sls, b, causal=causal)
    R.check(got, want, bound, str(case))
    assert torch.equal(got, prefill(sls, b, causal=causal))
    # a workspace of the caller's, filled with anything
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(got, prefill(sls, b, causal=causal, workspace=ws))


def test_prefill_cut_not_finite(sls):
    """The same as whole items: what a row does not see does not reach it."""
    b = R.make_batch([40], [5000], 4, 2, 64, 16, torch.bfloat16, seed=67)
    want, bound = R.attention(b)
    x = 4990                                      # seen from row 30 on
    b["v"][b["table"][0, x // 16].long(), x % 16, :, 9] = float("inf")
    got = prefill(sls, b)
    R.check(got[:30], want[:30], bound[:30])
    R.check(got[30:, :, :9], want[30:, :, :9], bound[30:, :, :9])
    assert torch.isinf(got[30:, :, 9]).all()


def test_workspaces_that_are_too_small(sls):
    b = R.make_batch([50], [10050], 28, 4, 128, 64, torch.bfloat16, seed=71)
    small = torch.empty(1024, dtype=torch.uint8, device="cuda")
    with pytest.raises(sls.SLSError) as e:
        prefill(sls, b, workspace=small)
    assert e.value.status == 3
    b = R.make_batch([1] * 70, [1000] * 70, 8, 8, 64, 16, torch.bfloat16, seed=73)
    with pytest.raises(sls.SLSError) as e:
        decode(sls, b, workspace=small)
    assert e.value.status == 3
    assert sls.attention_status() == 0


def test_prefill_same_bits_twice(sls):
    b = R.make_batch([500, 90], [900, 90], 28, 4, 128, 64, torch.bfloat16, seed=19)
    assert torch.equal(prefill(sls, b), prefill(sls, b))


def test_offsets_past_32_bits(sls):
    """A cache of more than 2^31 elements, the sequence in its last pages."""
    n, page, H, hd = 2100000, 16, 1, 128                  # 4.3e9 elements
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    k = torch.zeros(n, page, H, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n, page, H, hd, dtype=torch.bfloat16, device="cuda")
    b = R.make_batch([70], [95], 4, 1, 128, page, torch.bfloat16, seed=23)
    pages = 6
    src = b["table"][0, :pages].long()
    dst = torch.tensor([n - 1, 3, n - 2, 1100000, n - 7, 1050000], device="cuda")
    k[dst], v[dst] = b["k"][src], b["v"][src]
    b["table"][0, :pages] = dst.to(torch.int32)
    b["k"], b["v"] = k, v
    want, bound = R.attention(b)
    R.check(prefill(sls, b), want, bound)
    x = torch.randn(70, 6, hd, device="cuda").bfloat16()
    sls.qkv_append(x[:, :4], x[:, 4:5], x[:, 5:], k, v, b["table"], b["kv_lens"],
                   cu_seqlens=b["cu"])
    assert torch.equal(R.gather(k, b["table"][0], 95, page)[25:], x[:, 4:5])
    assert torch.equal(R.gather(v, b["table"][0], 95, page)[25:], x[:, 5:])
    b["new"], b["q"] = [1], b["q"][:1].contiguous()
    want, bound = R.attention(b)
    R.check(decode(sls, b), want, bound)


# ---------------------------------------------------------------------------
# decode
# ---------------------------------------------------------------------------

DECODE = [
    # m, Hq, Hkv, hd, page
    ([1], 1, 1, 64, 16),
    ([1, 2, 3], 28, 4, 128, 64),
    ([0, 5, 0, 64, 65], 14, 2, 64, 16),
    ([2061], 28, 4, 128, 64),
    ([20000], 40, 8, 128, 128),
    ([1, 8000, 17, 300], 32, 8, 128, 16),
    ([513], 16, 1, 128, 32),
    ([900, 31], 17, 1, 128, 32),                 # a group of 17: more than one block of rows
    ([900, 31], 128, 1, 64, 32),
    ([700, 255, 256, 257], 10, 2, 80, 32),
    ([333], 9, 3, 96, 16),
    ([400], 40, 40, 8, 16),
    ([100 + 7 * i for i in range(200)], 12, 12, 64, 32),
    ([3 * (i % 50) for i in range(1500)], 4, 2, 64, 16),
    ([5000], 8, 8, 128, 1024),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", DECODE)
def test_decode(sls, case, dtype):
    m, Hq, Hkv, hd, page = case
    b = R.make_batch([1] * len(m), m, Hq, Hkv, hd, page, dtype, seed=29)
    want, bound = R.attention(b)
    R.check(decode(sls, b), want, bound, str(case)[:80])


@pytest.mark.parametrize("order", ["tokens", "heads"])
def test_decode_strides(sls, order):
    m = [300, 1, 77]
    b = R.make_batch([1] * 3, m, 8, 2, 128, 32, torch.float16, seed=31, order=order)
    wide = torch.zeros(3, 13, 128, dtype=torch.float16, device="cuda")
    wide[:, 3:11] = b["q"]
    b["q"] = wide[:, 3:11]
    room = torch.full((3, 10, 136), 3.0, dtype=torch.float16, device="cuda")
    out = room[:, 1:9, :128]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode(sls, b, scale=0.05, out=out)
    side.synchronize()
    want, bound = R.attention(b, True, 0.05)
    R.check(out, want, bound)
    keep = torch.ones_like(room, dtype=torch.bool)
    keep[:, 1:9, :128] = False
    assert (room[keep] == 3.0).all()


def test_decode_bad_pages_read_as_zeros(sls):
    """A page number outside the cache reads as zeros (score 0, value 0)."""
    b = R.make_batch([1, 1], [100, 50], 4, 2, 64, 16, torch.bfloat16, seed=37)
    z = dict(b)
    z["k"], z["v"], z["table"] = b["k"].clone(), b["v"].clone(), b["table"].clone()
    for row, col in ((0, 2), (1, 3)):
        z["k"][b["table"][row, col].long()] = 0
        z["v"][b["table"][row, col].long()] = 0
        b["table"][row, col] = -1 if row else 1 << 30
    want, bound = R.attention(z)
    R.check(decode(sls, b), want, bound)
    R.check(prefill(sls, b), want, bound)


def test_decode_not_finite_values_stay_in_their_sequence(sls):
    b = R.make_batch([1] * 3, [200, 90, 300], 4, 2, 64, 16, torch.bfloat16, seed=41)
    want, bound = R.attention(b)
    b["v"][b["table"][1, 2].long(), 3] = float("nan")
    got = decode(sls, b)
    R.check(got[[0, 2]], want[[0, 2]], bound[[0, 2]])
    assert torch.isnan(got[1]).all()


def test_decode_same_bits_twice(sls):
    b = R.make_batch([1] * 9, [37 * i * i for i in range(9)], 28, 4, 128, 64, torch.bfloat16,
                     seed=43)
    assert torch.equal(decode(sls, b), decode(sls, b))


def test_decode_agrees_with_prefill_of_one(sls):
    b = R.make_batch([1] * 4, [600, 3, 1, 129], 28, 4, 128, 64, torch.bfloat16, seed=47)
    want, bound = R.attention(b)
    R.check(prefill(sls, b), want, bound)
    R.check(decode(sls, b), want, bound)


def test_graph_replay(sls):
    """The calls enqueue on the caller's stream only: a captured step replays."""
    b = R.make_batch([1] * 4, [600, 3, 1, 129], 28, 4, 128, 64, torch.bfloat16, seed=53)
    x = torch.randn(4, 28 + 8, 128, device="cuda").bfloat16()
    rope = sls.Rope.make(128)

    def step():
        q = sls.qkv_append(x[:, :28], x[:, 28:32], x[:, 32:], b["k"], b["v"], b["table"],
                           b["kv_lens"], rope=rope)
        return decode(sls, dict(b, q=q)), prefill(sls, dict(b, q=q))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    x.copy_(torch.randn(4, 28 + 8, 128, device="cuda"))
    g.replay()
    want = step()
    torch.cuda.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    assert sls.attention_status() == 0


# ---------------------------------------------------------------------------
# nothing to do
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("sequences", [0, 3])
def test_no_tokens(sls, sequences):
    """No new tokens, of no sequence or of some: empty results, an untouched cache."""
    b = R.make_batch([0] * sequences, [20] * sequences, 4, 2, 64, 16, torch.bfloat16, seed=83,
                     fill=1.0)
    k, v = b["k"].clone(), b["v"].clone()
    rows = b["k"].new_empty(0, 2, 64)
    out = sls.qkv_append(b["q"], rows, rows, b["k"], b["v"], b["table"], b["kv_lens"],
                         cu_seqlens=b["cu"])
    assert out.shape == (0, 4, 64) and prefill(sls, b).shape == (0, 4, 64)
    if sequences == 0:
        assert decode(sls, b).shape == (0, 4, 64)
    assert torch.equal(b["k"], k) and torch.equal(b["v"], v)
    assert sls.attention_status() == 0


def test_page_table_without_columns(sls):
    """Lengths are cut to what the table holds: rows without keys, which are zero."""
    b = R.make_batch([1, 1], [20, 5], 4, 2, 64, 16, torch.float16, seed=89)
    b["table"] = b["table"][:, :0].contiguous()
    for got in (prefill(sls, b), decode(sls, b)):
        assert torch.equal(got, torch.zeros_like(got))
    assert sls.attention_status() == 0
