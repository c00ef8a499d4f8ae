"""The calls that make the cache smaller (8-bit append, decode, prefill; attention weights;
eviction) against float64 statements of their definitions (tests/small_cache_ref.py), at
lengths, head layouts, blocks, strides and masks where a tiled kernel can go wrong.  Slots that
no sequence covers hold NaN (or the code -128) under NaN scales, so nothing but the covered ones
may reach a result."""
import math

import pytest
import torch

from tests import attention_ref as R
from tests import small_cache_ref as S

pytestmark = pytest.mark.gpu

CODES = [torch.int8, torch.float8_e4m3fn]
DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def batch(new, m, Hq, Hkv, hd, page, block, dtype, code, seed=1, **kw):
    return S.codes_of(R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed, **kw), code, block,
                      seed=seed)


def cache(b):
    return b["k"], b["v"], b["k_scale"], b["v_scale"], b["table"], b["kv_lens"]


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

APPEND = [
    # new, m, Hq, Hkv, hd, page, block, pairs, interleaved, norm, positions
    ([1], [1], 4, 1, 128, 16, 16, 64, False, True, True),
    ([1, 1, 1], [5, 700, 33], 28, 4, 128, 64, 64, 64, False, True, True),
    ([1] * 40, list(range(1, 41)), 8, 8, 64, 64, 32, 32, True, False, True),
    ([5, 0, 17, 130], [5, 9, 40, 1000], 14, 2, 64, 16, 16, 32, True, True, True),
    ([33, 8], [40, 8], 6, 3, 96, 32, 32, 48, False, False, True),
    ([33, 8], [40, 8], 6, 3, 96, 32, 16, 12, False, True, True),     # halves of 12: no whole vectors
    ([20, 7], [50, 7], 10, 2, 80, 16, 16, 9, True, True, False),     # an odd number of pairs
    ([9], [4], 4, 4, 16, 16, 16, 8, False, True, True),              # more tokens than cache places
    ([200], [264], 8, 8, 48, 1024, 128, 0, False, True, True),       # no rotation
    ([300, 500], [4000, 501], 40, 8, 128, 128, 128, 64, True, False, True),
    ([700, 1, 64], [700, 129, 64], 2, 1, 128, 128, 64, 40, False, True, True),
    ([1, 2, 0], [50, 7, 9], 10, 2, 80, 16, 16, 9, False, True, True),   # few tokens, odd halves
    ([1, 1, 3], [50, 7, 20], 40, 8, 128, 32, 16, 0, False, True, False),  # a norm alone
    ([2, 1], [2, 128], 3, 3, 32, 128, 128, 5, True, False, False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", APPEND)
def test_append(sls, case, code, dtype):
    new, m, Hq, Hkv, hd, page, block, pairs, inter, norm, use_pos = case
    # the cache as it was before: only the earlier tokens are there
    old = [max(0, y - x) for x, y in zip(new, m)]
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=3)
    for s, (o, y) in enumerate(zip(old, m)):
        for i in range(o, y):
            b["k"][b["table"][s, i // page].long(), i % page] = math.nan
            b["v"][b["table"][s, i // page].long(), i % page] = math.nan
    b = S.codes_of(b, code, block, seed=4)
    T = sum(new)
    g = torch.Generator("cuda").manual_seed(3)
    qkv = torch.randn(T, Hq + 2 * Hkv, hd, generator=g, device="cuda")
    qkv = (qkv * torch.exp(0.5 * torch.randn(T, 1, 1, generator=g, device="cuda"))).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    qw = kw = None
    if norm:
        qw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
        kw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
    pos = torch.randint(0, 131072, (T,), generator=g, device="cuda", dtype=torch.int32)
    idx = torch.cat([torch.arange(y - x, y) for x, y in zip(new, m)]).cuda()
    pos = pos if use_pos else None
    f = sls.Rope.make(max(2, 2 * pairs), base=1e6).inv_freq[:pairs].contiguous()
    rope = sls.Rope(f, interleaved=inter, scale=1.25) if pairs else None
    at = (f if pairs else None, inter, 1.25, pos if use_pos else idx)
    qo, qe = S.turned(q, qw, 1e-5, *at)
    ky, ke = S.turned(k, kw, 1e-5, *at)
    K = S.append(b, "k", ky, ke)
    V = S.append(b, "v", v.double(), torch.zeros_like(ke[:, :1]).expand(-1, Hkv, -1))
    old_codes = {x: b[x].clone() for x in "kv"}
    twin = dict(b, **{x: b[x].clone() for x in ("k", "v", "k_scale", "v_scale")})
    got = sls.qkv_append_q8(q, k, v, *cache(b), cu_seqlens=b["cu"], positions=pos, q_weight=qw,
                            k_weight=kw, eps=1e-5, rope=rope)
    S.check(got, qo, qe + R.U[dtype] * qo.abs() + R.TINY[dtype], "q")
    for x, (val, err, sc) in (("k", K), ("v", V)):
        live = ~torch.isnan(sc)
        assert torch.equal(~torch.isnan(b[x + "_scale"]), live), x
        off = (b[x + "_scale"].double() / sc - 1)[live].nonzero()
        assert off.numel() == 0, f"{x}: {off.shape[0]} of {int(live.sum())} scales"
        hole = torch.isnan(val)
        now = S.values(b, x)
        assert torch.equal(torch.isnan(now), hole), x
        S.check(now.masked_fill(hole, 0), val.masked_fill(hole, 0), err.masked_fill(hole, 0), x)
        # what no sequence covers is left as it was
        raw = b[x].view(torch.uint8)[hole]
        assert torch.equal(raw, old_codes[x].view(torch.uint8)[hole]), x
    # in place
    again = sls.qkv_append_q8(q, k, v, *cache(twin), cu_seqlens=b["cu"], positions=pos, q_weight=qw,
                              k_weight=kw, eps=1e-5, rope=rope, out=q)
    assert again is q and torch.equal(q, got)
    assert all(torch.equal(twin[x].view(torch.uint8), b[x].view(torch.uint8)) for x in "kv")


@pytest.mark.parametrize("code", CODES)
def test_append_token_by_token(sls, code):
    """Tokens that come one by one, ever larger: the block's scale grows with them and what was
    there is rounded again each time; without growth nothing earlier changes."""
    hd, H, page = 64, 2, 16
    b = R.make_batch([1], [40], H, H, hd, page, torch.float16, seed=9)
    b["k"].fill_(math.nan), b["v"].fill_(math.nan)
    b = S.codes_of(b, code, 16)
    g = torch.Generator("cuda").manual_seed(1)
    scales = []
    for i in range(40):
        size = 2.0 ** min(i, 8)
        x = (torch.randn(1, 3 * H, hd, generator=g, device="cuda") * size).half()
        b["m"] = [i + 1]
        b["kv_lens"].fill_(i + 1)
        zero = torch.zeros(1, H, hd, dtype=torch.float64, device="cuda")
        K = S.append(b, "k", x[:, H:2 * H].double(), zero)
        V = S.append(b, "v", x[:, 2 * H:].double(), zero)
        before = b["k"].clone()
        sls.qkv_append_q8(x[:, :H], x[:, H:2 * H], x[:, 2 * H:], *cache(b))
        for name, (val, err, sc) in (("k", K), ("v", V)):
            hole = torch.isnan(val)
            assert torch.equal(torch.isnan(S.values(b, name)), hole)
            S.check(S.values(b, name).masked_fill(hole, 0), val.masked_fill(hole, 0),
                    err.masked_fill(hole, 0), name)
            live = ~torch.isnan(sc)
            assert torch.equal(b[name + "_scale"][live].double(), sc[live])
        pg = int(b["table"][0, i // page])
        scales.append(b["k_scale"][pg, 0].clone())
        if i % page and torch.equal(scales[-1], scales[-2]):
            was, now = before.view(torch.uint8)[pg, :i % page], b["k"].view(torch.uint8)[pg, :i % page]
            assert torch.equal(was, now)


@pytest.mark.parametrize("code", CODES)
def test_append_values_that_are_not_finite(sls, code):
    hd, page = 32, 16
    b = R.make_batch([20], [20], 1, 1, hd, page, torch.bfloat16, seed=2)
    b["k"].fill_(math.nan), b["v"].fill_(math.nan)
    b = S.codes_of(b, code, 16)
    x = torch.randn(20, 3, hd, device="cuda").bfloat16()
    x[3, 2, 5], x[4, 2, 6], x[5, 2, 7] = math.inf, -math.inf, math.nan
    x[17, 2] = 0.0
    x[18, 2] = math.inf
    sls.qkv_append_q8(x[:, :1], x[:, 1:2], x[:, 2:], *cache(b), cu_seqlens=b["cu"])
    pg = b["table"][0].long()
    v = S.index8(b["v"], pg[0]).float()[:, 0]
    most = S.MOST[code]
    assert v[3, 5] == most and v[4, 6] == -most
    assert (v[5, 7] == 0) if code == torch.int8 else torch.isnan(v[5, 7])
    y = x[:16, 2].double()
    y[3, 5] = y[4, 6] = y[5, 7] = 0.0
    s = S.power(y.abs().max(), code)
    assert b["v_scale"][pg[0], 0, 0].double() == s
    fin = x[:16, 2].isfinite()
    off = (v.double() * s - x[:16, 2].double()).abs()[fin]
    assert (off <= S.half_step(x[:16, 2].double() / s, code)[fin] * s).all()


def test_append_skips_what_has_no_place(sls):
    """Tokens past the last sequence, page numbers outside the cache and indices past the table:
    nothing is written, the queries are."""
    b = batch([4, 4], [20, 300], 4, 2, 64, 16, 16, torch.bfloat16, torch.int8, seed=7)
    cols = b["table"].shape[1]
    b["kv_lens"][1] = cols * 16 + 2        # the last two new tokens lie past the table
    b["table"][0, 1] = -5                  # sequence 0's second page is none
    b["table"][1, cols - 1] = 1 << 30
    x = torch.randn(11, 8, 64, device="cuda").bfloat16()
    before = [t.clone() for t in cache(b)[:4]]
    out = sls.qkv_append_q8(x[:, :4], x[:, 4:6], x[:, 6:], *cache(b), cu_seqlens=b["cu"])
    assert torch.equal(out, x[:, :4])
    for a, c in zip(before, cache(b)):
        assert torch.equal(a.view(torch.uint8), c.view(torch.uint8))


# ---------------------------------------------------------------------------
# attention over codes
# ---------------------------------------------------------------------------

DECODE = [
    # m, Hq, Hkv, hd, page, block
    ([1], 4, 1, 128, 16, 16),
    ([2061], 28, 4, 128, 64, 64),
    ([0, 5, 700, 33, 32, 31, 64], 14, 2, 64, 16, 16),
    ([1, 17, 513], 6, 3, 96, 32, 16),
    ([100, 40], 34, 2, 80, 128, 32),           # 17 query heads a key head: two tiles
    ([300] * 30, 12, 12, 64, 32, 32),
    ([4000, 3], 128, 1, 16, 1024, 128),
    ([9000, 100, 5000], 40, 8, 128, 128, 128),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", DECODE)
def test_decode(sls, case, code, dtype):
    m, Hq, Hkv, hd, page, block = case
    b = batch([1] * len(m), m, Hq, Hkv, hd, page, block, dtype, code, seed=5)
    want, bound = R.attention(S.plain(b), causal=False)
    S.check(sls.attention_decode_q8(b["q"], *cache(b)), want, bound, "decode")


@pytest.mark.parametrize("code", CODES)
def test_decode_scales_far_apart(sls, code):
    """Blocks whose values' scales differ by up to 2^40, in both orders of size."""
    for sign in (1, -1):
        b = batch([1, 1], [256, 200], 8, 2, 64, 16, 16, torch.bfloat16, code, seed=6)
        for x, far in (("k", 1), ("v", 40)):
            for s in range(2):
                for i in range(int(b["m"][s] + 15) // 16):
                    pg = int(b["table"][s, i])
                    b[x + "_scale"][pg] *= 2.0 ** (sign * far * (i - 8) // 8)
        want, bound = R.attention(S.plain(b), causal=False)
        S.check(sls.attention_decode_q8(b["q"], *cache(b)), want, bound, "decode")


def test_decode_zero_scales_and_pages_outside(sls):
    b = batch([1, 1], [64, 50], 4, 2, 64, 16, 16, torch.float16, torch.int8, seed=6)
    b["v_scale"][b["table"][0, 0].long()] = 0.0
    b["v_scale"][b["table"][0, 2].long()] = 0.0
    for i in range(4):
        b["k_scale"][b["table"][1, i].long()] = 0.0
        b["v_scale"][b["table"][1, i].long()] = 0.0
    want, bound = R.attention(S.plain(b), causal=False)
    S.check(sls.attention_decode_q8(b["q"], *cache(b)), want, bound, "decode")
    # a page outside the cache reads as zeros
    bad = dict(b, table=b["table"].clone())
    pg = int(b["table"][0, 1])
    bad["table"][0, 1] = 1 << 29
    for x in "kv":
        b[x].view(torch.uint8)[pg] = 0
        b[x + "_scale"][pg] = 0
    want, bound = R.attention(S.plain(b), causal=False)
    S.check(sls.attention_decode_q8(b["q"], *cache(bad)), want, bound, "decode")


PREFILL = [
    # new, m, Hq, Hkv, hd, page, block, causal
    ([1], [1], 4, 1, 128, 16, 16, True),
    ([137], [137], 28, 4, 128, 64, 64, True),
    ([5, 0, 300, 33], [5, 9, 700, 1000], 14, 2, 64, 16, 16, True),
    ([40, 9], [50, 4], 6, 3, 96, 32, 32, True),          # rows that see no key
    ([64, 3], [200, 77], 10, 2, 80, 128, 64, False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", PREFILL)
def test_prefill(sls, case, code, dtype):
    new, m, Hq, Hkv, hd, page, block, causal = case
    b = batch(new, m, Hq, Hkv, hd, page, block, dtype, code, seed=8)
    want, bound = R.attention(S.plain(b), causal=causal)
    got = sls.attention_prefill_q8(b["q"], *cache(b), b["cu"], causal=causal)
    S.check(got, want, bound, "prefill")


def test_prefill_wide_table_and_shared_pages(sls):
    """A table of more entries than the cache has pages: the pages are written out under their
    own numbers; two sequences share their first pages."""
    b = batch([20, 30], [64, 80], 4, 2, 64, 16, 16, torch.bfloat16, torch.int8, seed=3)
    wide = torch.full((2, 40), 1 << 20, dtype=torch.int32, device="cuda")
    wide[:, :b["table"].shape[1]] = b["table"]
    wide[1, :2] = wide[0, :2]
    b["table"] = wide
    want, bound = R.attention(S.plain(b))
    S.check(sls.attention_prefill_q8(b["q"], *cache(b), b["cu"]), want, bound, "prefill")


# ---------------------------------------------------------------------------
# weights
# ---------------------------------------------------------------------------

WEIGHTS = [
    # new, m, Hq, Hkv, hd, page, block, causal
    ([1], [1], 4, 1, 128, 16, 16, True),
    ([1] * 5, [5, 700, 33, 0, 256], 28, 4, 128, 64, 64, True),
    ([5, 0, 300, 33], [5, 9, 700, 1000], 14, 2, 64, 16, 16, True),   # several blocks of rows
    ([40, 9], [50, 4], 6, 3, 96, 32, 32, True),                     # rows that see no key
    ([64, 3], [200, 77], 10, 2, 80, 128, 64, False),
    ([32], [3000], 16, 1, 64, 128, 32, True),
    ([2, 1, 1], [257, 255, 600], 16, 8, 48, 32, 16, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("code", [None] + CODES)
@pytest.mark.parametrize("case", WEIGHTS)
def test_weights(sls, case, code, dtype):
    new, m, Hq, Hkv, hd, page, block, causal = case
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=11)
    p, scale = b, None
    if code is not None:
        b = S.codes_of(b, code, block, seed=11)
        p, scale = S.plain(b), b["k_scale"]
    g = torch.Generator("cuda").manual_seed(2)
    w = torch.rand(b["k"].shape[0], Hkv, page, generator=g, device="cuda")
    want, bound = S.weights(p, w, causal=causal)
    first = w.clone()
    got = sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                                k_scale=scale, causal=causal)
    assert got is w
    S.check(w, want, bound, "weights")
    # the same call gives the same bits
    sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], first, cu_seqlens=b["cu"],
                          k_scale=scale, causal=causal)
    assert torch.equal(first, w)


@pytest.mark.parametrize("rows", [1, 16, 40])
def test_weights_of_scores_far_from_zero(sls, rows):
    """Scores of 423 that differ by 0 or 3.33 and are exact (one element of a query and a code
    each): what is left are the exponents' roundings, which go by the distance from the maximum and
    not by the score.  In units of 2^-24: an exponent of at most 4.8 is off by 2 for the rounded
    factor and 1 for its own rounding, all of that times 4.8 log(2), and its power by 4: 14, for the
    weight and for the sum; sums of earlier tokens are taken to a larger maximum in at most three
    places, 14 each; their additions and products are at most 16, a weight's own and its column's 16:
    102."""
    m, page, block, scale = 300, 64, 32, 1.6661376953125
    k = torch.zeros(5, page, 1, 64, dtype=torch.int8, device="cuda")
    idx = torch.arange(5 * page, device="cuda").view(5, page)
    k[:, :, 0, 0] = torch.where((idx < 128) | (idx % 3 == 0), 126, 127).to(torch.int8)
    ones = torch.ones(5, page // block, 1, device="cuda")
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([m], dtype=torch.int32, device="cuda")
    q = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 2
    w = torch.zeros(5, 1, page, device="cuda")
    sls.attention_weights(q, k, table, lens, w, torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                          k_scale=ones, causal=False, scale=scale)
    s = 2 * k[:, :, 0, 0].double().flatten()[:m] * scale
    want = rows * torch.softmax(s, 0)
    error = ((w.flatten()[:m].double() - want).abs() / want).max().item()
    assert error <= 102 * 2 ** -24, error * 2 ** 24


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------

EVICT = [
    # m, Hkv, hd, page, block, keep, first, last
    ([100], 1, 128, 16, 16, 10, 2, 3),
    ([0, 5, 700, 33, 64], 2, 64, 16, 16, 32, 4, 8),
    ([300, 200], 3, 96, 32, 32, 131, 0, 0),
    ([1500, 40, 1100], 2, 48, 128, 64, 1030, 1, 64),
    ([90, 17], 2, 16, 64, 64, 16, 8, 8),             # no room for others
    ([90, 17], 2, 16, 1024, 128, 0, 0, 0),
    ([50, 20], 1, 32, 16, 16, 49, 0, 1),
]


@pytest.mark.parametrize("code", [None] + CODES)
@pytest.mark.parametrize("case", EVICT)
def test_evict(sls, case, code):
    m, Hkv, hd, page, block, keep, first, last = case
    b = R.make_batch([1] * len(m), m, Hkv, Hkv, hd, page, torch.bfloat16, seed=12)
    if code is not None:
        b = S.codes_of(b, code, block, seed=12)
    g = torch.Generator("cpu").manual_seed(4)
    w = torch.rand(b["k"].shape[0], Hkv, page, generator=g)
    w = (w * 40).round() / 8 - 1               # many equal ones, negative ones
    w[torch.rand(w.shape, generator=g) < 0.05] = math.nan
    w[torch.rand(w.shape, generator=g) < 0.05] = -0.0
    w[torch.rand(w.shape, generator=g) < 0.02] = math.inf
    w[torch.rand(w.shape, generator=g) < 0.02] = -math.inf
    host = {k: (v.cpu() if torch.is_tensor(v) else v) for k, v in b.items()}
    want = S.evict(host, w, keep, first, last)
    w = w.cuda()
    scales = (None, None) if code is None else (b["k_scale"], b["v_scale"])
    kept = sls.cache_evict(b["k"], b["v"], b["table"], b["kv_lens"], w, keep, first=first,
                           last=last, k_scale=scales[0], v_scale=scales[1])
    assert torch.equal(kept.cpu(), want["kept"])
    assert torch.equal(b["kv_lens"].cpu(), want["lens"])
    assert torch.equal(torch.nan_to_num(w.cpu(), nan=77.0), torch.nan_to_num(want["w"], nan=77.0))
    for x, t in zip("kv", scales):
        raw = b[x].cpu().view(torch.int16 if code is None else torch.uint8)
        assert torch.equal(raw, want[x]), x
        if t is not None:
            assert torch.equal(torch.nan_to_num(t.cpu(), nan=-1.0),
                               torch.nan_to_num(want[x + "_scale"], nan=-1.0)), x
