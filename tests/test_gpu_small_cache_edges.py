"""The calls that make the cache smaller at the edges of their numbers: keys of zeros behind a norm,
scales below zero, values that are far apart in size."""
import pytest
import torch

from tests import attention_ref as R
from tests import small_cache_ref as S
from tests.test_gpu_small_cache import CODES, batch, cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def only_earlier(new, m, H, hd, page, block, dtype, code, seed):
    """A cache that holds the tokens before the new ones."""
    b = R.make_batch(new, m, H, H, hd, page, dtype, seed=seed)
    for s, (n, length) in enumerate(zip(new, m)):
        for i in range(max(0, length - n), length):
            for x in "kv":
                b[x][b["table"][s, i // page].long(), i % page] = float("nan")
    return S.codes_of(b, code, block, seed=seed)


def appended(sls, b, qkv, H, norm, rope, f, inter, eps):
    """Appends and compares codes and scales with the definition."""
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    idx = torch.cat([torch.arange(m - n, m) for n, m in zip(b["new"], b["m"])]).cuda()
    ky, ke = S.turned(k, norm, eps, f, inter, 1.0, idx)
    want = {"k": S.append(b, "k", ky, ke), "v": S.append(b, "v", v.double(), 0.0 * ke)}
    out = sls.qkv_append_q8(q, k, v, *cache(b), cu_seqlens=b["cu"], q_weight=norm, k_weight=norm,
                            eps=eps, rope=rope)
    for x, (val, err, sc) in want.items():
        live = ~torch.isnan(sc)
        assert torch.equal(b[x + "_scale"][live].double(), sc[live]), x
        hole = torch.isnan(val)
        now = S.values(b, x)
        assert torch.equal(torch.isnan(now), hole), x
        S.check(now.masked_fill(hole, 0), val.masked_fill(hole, 0), err.masked_fill(hole, 0), x)
    return out


TURNS = [(32, False), (32, True), (12, False), (0, False)]   # pairs, side by side


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("pairs,inter", TURNS)
@pytest.mark.parametrize("new,m,zero", [
    ([1, 1, 1], [1, 17, 40], [0, 1, 2]),              # a token that opens a block, or joins one
    ([40, 20], [40, 52], list(range(16)) + [20, 57]),  # a block of nothing else; one among others
])
def test_append_of_zero_keys_behind_a_norm(sls, new, m, zero, pairs, inter, code):
    """Their norm is 1 / sqrt(eps), their block's scale 2^-126: the codes are zeros, and stay so when
    the block takes a token of some size."""
    H, hd, page, block = 4, 64, 32, 16
    b = only_earlier(new, m, H, hd, page, block, torch.bfloat16, code, seed=31)
    g = torch.Generator("cuda").manual_seed(5)
    qkv = torch.randn(sum(new), 3 * H, hd, generator=g, device="cuda").bfloat16()
    qkv[torch.tensor(zero), H:2 * H] = 0
    norm = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16()
    f = sls.Rope.make(64, base=1e4).inv_freq[:pairs].contiguous() if pairs else None
    rope = sls.Rope(f, interleaved=inter) if pairs else None
    q = appended(sls, b, qkv, H, norm, rope, f, inter, 1e-6)

    def zeros():
        t0 = 0
        for s, (n, length) in enumerate(zip(new, m)):
            for t in zero:
                if t0 <= t < t0 + n:
                    i = length - n + t - t0
                    at = S.index8(b["k"], b["table"][s, i // page].long(), i % page)
                    assert not at.float().any()
            t0 += n

    zeros()
    last = q[b["cu"][1:].long() - 1]
    want, bound = R.attention(dict(S.plain(b), q=last, new=[1] * len(m)), causal=False)
    S.check(sls.attention_decode_q8(last, *cache(b)), want, bound, "decode")
    # the next token
    b.update(new=[1] * len(m), m=[x + 1 for x in m],
             cu=torch.arange(len(m) + 1, dtype=torch.int32, device="cuda"))
    b["kv_lens"] += 1
    more = torch.randn(len(m), 3 * H, hd, generator=g, device="cuda").bfloat16()
    appended(sls, b, more, H, norm, rope, f, inter, 1e-6)
    zeros()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("n", [1, 16])
def test_append_of_the_smallest_keys_behind_a_norm(sls, n, code):
    """Keys of 2^-128, whose norm of 1000 and whose block's factor of 2^124 meet past float32."""
    H, hd = 4, 64
    b = only_earlier([n], [n], H, hd, 32, 16, torch.bfloat16, code, seed=7)
    g = torch.Generator("cuda").manual_seed(6)
    qkv = torch.randn(n, 3 * H, hd, generator=g, device="cuda")
    qkv[:, H:2 * H] = qkv[:, H:2 * H].sign() * 2.0 ** -128
    appended(sls, b, qkv.bfloat16(), H, torch.ones(hd, device="cuda").bfloat16(), None, None, False,
             1e-6)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("H,hd", [(1, 128), (3, 64), (5, 128), (7, 64)])
def test_append_where_keys_and_values_share_a_block_of_threads(sls, H, hd, block, code):
    """Few blocks, so that several warps have a head: the last key head's beside the first value
    head's, some without a head at the end.  Right, and the same bits twenty times."""
    new, m = [150, 70], [150, 211]
    b = only_earlier(new, m, H, hd, 128, block, torch.bfloat16, code, seed=61)
    g = torch.Generator("cuda").manual_seed(5)
    qkv = torch.randn(sum(new), 3 * H, hd, generator=g, device="cuda").bfloat16()
    norm = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16()
    rope = sls.Rope.make(hd)
    names = ("k", "v", "k_scale", "v_scale")
    before = {x: b[x].clone() for x in names}
    appended(sls, b, qkv, H, norm, rope, rope.inv_freq, False, 1e-6)
    for _ in range(20):
        c = dict(b, **{x: before[x].clone() for x in names})
        sls.qkv_append_q8(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], *cache(c), cu_seqlens=b["cu"],
                          q_weight=norm, k_weight=norm, eps=1e-6, rope=rope)
        assert all(torch.equal(c[x].view(torch.uint8), b[x].view(torch.uint8)) for x in names)


@pytest.mark.parametrize("code", CODES)
def test_append_and_decode_of_a_padded_batch(sls, code):
    """Places of a batch without a sequence (length 0, a table row of any numbers) take and change
    nothing; the others are as without them."""
    m, H, hd, page, block = [9, 40, 17], 4, 64, 32, 16
    b = only_earlier([1] * 3, m, H, hd, page, block, torch.bfloat16, code, seed=71)
    g = torch.Generator("cuda").manual_seed(8)
    qkv = torch.randn(7, 3 * H, hd, generator=g, device="cuda").bfloat16()
    real = torch.tensor([1, 2, 5], device="cuda")
    table = torch.randint(-9, 99, (7, b["table"].shape[1]), device="cuda").int()
    table[real] = b["table"]
    lens = torch.zeros(7, dtype=torch.int32, device="cuda")
    lens[real] = b["kv_lens"]
    names = ("k", "v", "k_scale", "v_scale")
    c = dict(b, table=table, kv_lens=lens, **{x: b[x].clone() for x in names})
    rope = sls.Rope.make(hd)
    out = []
    for d, x in ((b, qkv[real]), (c, qkv)):
        q = sls.qkv_append_q8(x[:, :H], x[:, H:2 * H], x[:, 2 * H:], *cache(d), rope=rope)
        w = torch.zeros(b["k"].shape[0], H, page, device="cuda")
        sls.attention_weights(q, d["k"], d["table"], d["kv_lens"], w, k_scale=d["k_scale"])
        out.append((q, sls.attention_decode_q8(q, *cache(d)), w))
    assert all(torch.equal(b[x].view(torch.uint8), c[x].view(torch.uint8)) for x in names)
    assert torch.equal(out[0][0], out[1][0][real])
    rest = torch.tensor([0, 3, 4, 6], device="cuda")
    assert not out[1][1][rest].any()
    want, bound = R.attention(dict(S.plain(b), q=out[0][0]), causal=False)
    S.check(out[1][1][real], want, bound, "decode")
    sums, err = S.weights(dict(S.plain(b), q=out[0][0]), torch.zeros_like(out[1][2]))
    S.check(out[1][2], sums, err, "weights")


# ---------------------------------------------------------------------------
# scales of either sign
# ---------------------------------------------------------------------------

def turned_over(b, seed):
    """The same values with the codes and scales of some blocks negated: all of sequence 0's, half of
    the others'."""
    out = dict(b)
    g = torch.Generator("cpu").manual_seed(seed)
    for x in "kv":
        sc = b[x + "_scale"]
        over = torch.rand(sc.shape, generator=g).to(sc.device) < 0.5
        over[b["table"][0][b["table"][0] < sc.shape[0]].long()] = True
        rows = over.repeat_interleave(b["block"], 1)[..., None]
        c = b[x].view(torch.uint8)
        neg = (-b[x]).view(torch.uint8) if b[x].dtype == torch.int8 else c ^ 0x80
        out[x] = torch.where(rows, neg, c).view(b[x].dtype)
        out[x + "_scale"] = torch.where(over, -sc, sc)
    return out


@pytest.mark.parametrize("code", CODES)
def test_scales_below_zero_attended(sls, code):
    new, m, page, block = [3, 20, 1], [70, 200, 900], 32, 16
    b = batch(new, m, 8, 2, 64, page, block, torch.bfloat16, code, seed=41)
    t = turned_over(b, 1)
    want, bound = R.attention(S.plain(b))
    S.check(sls.attention_prefill_q8(b["q"], *cache(t), b["cu"]), want, bound, "prefill")
    w = torch.zeros(b["k"].shape[0], 2, page, device="cuda")
    sums, err = S.weights(S.plain(b), w)
    sls.attention_weights(b["q"], t["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                          k_scale=t["k_scale"])
    S.check(w, sums, err, "weights")
    for many in (1, 40):       # clusters, and parts with pieces
        last = b["q"][b["cu"][1:].long() - 1].repeat(many, 1, 1)
        big = {k: t[k].repeat(many, 1) if k == "table" else t[k].repeat(many) for k in ("table", "kv_lens")}
        ref = dict(S.plain(b), q=last[:3], new=[1] * 3)
        want, bound = R.attention(ref, causal=False)
        got = sls.attention_decode_q8(last, t["k"], t["v"], t["k_scale"], t["v_scale"], big["table"],
                                      big["kv_lens"])
        S.check(got, want.repeat(many, 1, 1), bound.repeat(many, 1, 1), "decode")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("size", [0.01, 100.0])
@pytest.mark.parametrize("n", [1, 12])
def test_scales_below_zero_appended_to(sls, n, size, code):
    """A block that holds earlier tokens takes the size of its scale, and their codes its sign."""
    new, m, H, hd, page, block = [n] * 3, [n + 5, n + 27, n + 44], 4, 64, 32, 16
    b = only_earlier(new, m, H, hd, page, block, torch.bfloat16, code, seed=43)
    t = turned_over(b, 2)
    g = torch.Generator("cuda").manual_seed(5)
    x = (size * torch.randn(sum(new), 3 * H, hd, generator=g, device="cuda")).bfloat16()
    for c in (b, t):
        sls.qkv_append_q8(x[:, :H], x[:, H:2 * H], x[:, 2 * H:], *cache(c), cu_seqlens=b["cu"])
    for i in "kv":
        assert torch.equal(S.values(t, i).nan_to_num(7.0), S.values(b, i).nan_to_num(7.0)), i
        for s, length in enumerate(m):
            at = b["table"][s, (length - 1) // page].long(), (length - 1) % page // block
            assert torch.equal(t[i + "_scale"][at], b[i + "_scale"][at])


@pytest.mark.parametrize("code", CODES)
def test_scales_below_zero_evicted(sls, code):
    m, page, block, keep = [300, 20, 90], 32, 16, 41
    b = batch([1] * 3, m, 2, 2, 64, page, block, torch.bfloat16, code, seed=44)
    t = turned_over(b, 3)
    t["kv_lens"] = b["kv_lens"].clone()
    w = torch.rand(b["k"].shape[0], 2, page, device="cuda")
    got = []
    for c in (b, t):
        got.append(sls.cache_evict(c["k"], c["v"], c["table"], c["kv_lens"], w.clone(), keep, first=3,
                                   last=9, k_scale=c["k_scale"], v_scale=c["v_scale"]))
    assert torch.equal(*got)
    for i in "kv":
        a, z = S.values(b, i), S.values(t, i)
        for s, length in enumerate(m):
            n = min(length, keep)
            assert torch.equal(R.gather(a, b["table"][s], n, page), R.gather(z, b["table"][s], n, page))


# ---------------------------------------------------------------------------
# values far apart
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("B", [2, 64])                  # clusters, and parts with pieces
@pytest.mark.parametrize("where", [0, 1, 18, 37])       # block of sixteen among 37.5
def test_decode_of_large_values_that_one_head_sees(sls, where, B, code):
    """A block of values 2^40 times the others', which one query head of a key head looks at and the
    other (its weights there 2^-60 and less) does not: the other's result keeps its bits."""
    H, hd, m, page = 8, 64, 600, 16
    b = batch([1] * B, [m] * B, 2 * H, H, hd, page, 16, torch.bfloat16, code, seed=where)
    g = torch.Generator("cuda").manual_seed(9)
    u = torch.randn(B, H, hd, generator=g, device="cuda").sign()
    b["q"] = torch.stack([2 * u, -2 * u], 2).view(B, 2 * H, hd).bfloat16()
    used = min(16, m - 16 * where)
    for s in range(B):
        pg = int(b["table"][s, where])
        b["k"].view(torch.uint8)[pg, :used] = (96 * u[s]).to(code).view(torch.uint8)
        b["k_scale"][pg, 0] = 2.0 ** -5
        b["v_scale"][pg, 0] *= 2.0 ** 40
    want, bound = R.attention(S.plain(b), causal=False)
    # R.attention counts a float16 weight's 11 bits, not its least step (its 16-bit weights of bfloat16
    # have none): a weight times its value's scale, in units U of its head, is off by half of 2^-24; times
    # code and unit, over a sum of at least 2^15 (the largest weight is 2^15): 2^-40 U |code| a token.  U
    # is at most 16 times the scales that the head needs, rounded up to a power of two: 32 of the largest
    # scale, that of the block left out where the head's weights there, below 2^-60, need less than 1 / 16
    # of it.  (An element that is 0 where the head looks shows this: what is left of 600 tokens of 2^-30.)
    tiny = torch.zeros_like(bound)
    for s in range(B):
        pages = b["table"][s, :-(-m // page)].long()
        sc = b["v_scale"][pages, 0].double()                                   # blocks x key heads
        codes = torch.nan_to_num(S.values(b, "v")[pages], nan=0.0) / sc[:, None, :, None]
        total = codes.abs().sum((0, 1))                                       # key heads x elements
        other = torch.cat([sc[:where], sc[where + 1:]]).amax(0)
        unit = 32 * torch.stack([sc.amax(0), other], 1)                       # key heads x query heads
        tiny[s] = (2.0 ** -40 * unit[:, :, None] * total[:, None]).view(2 * H, hd)
    S.check(sls.attention_decode_q8(b["q"], *cache(b)), want, bound + tiny, "decode")


# ---------------------------------------------------------------------------
# eviction that leaves no choice
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("lengths", [[3000], [20000, 70, 9000], [131072], [400000]])
@pytest.mark.parametrize("first,last", [(4, 60), (0, 2049), (33, 0), (0, 0)])
def test_evict_to_the_first_and_last(sls, lengths, first, last):
    """No weight decides: sinks and a recent window stay, or nothing, by clusters of every size (two
    to eight CTAs for three sequences and for one) and past what they hold."""
    page, Hkv, hd, keep = 128, 2, 16, first + last
    B, per = len(lengths), [-(-m // page) for m in lengths]
    g = torch.Generator("cuda").manual_seed(sum(lengths))
    table = torch.zeros(B, max(per), dtype=torch.int32, device="cuda")
    order = torch.randperm(sum(per), generator=g, device="cuda").int()
    for s in range(B):
        table[s, :per[s]] = order[sum(per[:s]):sum(per[:s + 1])]
    n = sum(per)
    k = torch.randint(-99, 99, (n, page, Hkv, hd), generator=g, device="cuda").half()
    v = torch.randint(-99, 99, (n, page, Hkv, hd), generator=g, device="cuda").half()
    w = torch.rand(n, Hkv, page, generator=g, device="cuda") + 1
    old = [t.clone() for t in (k, v, w.transpose(1, 2)[..., None])]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kept = sls.cache_evict(k, v, table, lens, w, keep, first=first, last=last)
    assert lens.tolist() == [min(m, keep) for m in lengths]
    for s, m in enumerate(lengths):
        i = torch.arange(m, device="cuda")
        stay = i if m <= keep else torch.cat([i[:first], i[m - last:]])
        want = torch.full((keep,), -1, device="cuda")
        want[:stay.numel()] = stay
        assert (kept[s].long() == want).all()
        for a, b in zip(old, (k, v, w.transpose(1, 2)[..., None])):
            a, b = R.gather(a, table[s], m, page), R.gather(b, table[s], m, page)
            assert torch.equal(b[:stay.numel()], a[stay])
        if m > keep:
            assert not b[keep:].any()


# ---------------------------------------------------------------------------
# weights
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("code", [None] + CODES)
def test_weights_repeat_themselves(sls, code):
    """CTAs that go through several tiles of tokens, of one tile of rows or two, and over the ends of
    heads: right, and the same bits a hundred times."""
    new, m, Hq, Hkv, hd, page = [24, 40, 20], [14000, 9000, 5000], 16, 4, 64, 64
    b = R.make_batch(new, m, Hq, Hkv, hd, page, torch.bfloat16, seed=51)
    p, scale = b, None
    if code is not None:
        b = S.codes_of(b, code, 32, seed=51)
        p, scale = S.plain(b), b["k_scale"]
    zero = torch.zeros(b["k"].shape[0], Hkv, page, device="cuda")
    want, bound = S.weights(p, zero)
    sums = []
    for _ in range(100):
        sums.append(sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], zero.clone(),
                                          cu_seqlens=b["cu"], k_scale=scale))
    S.check(sums[0], want, bound, "weights")
    assert all(torch.equal(sums[0], w) for w in sums[1:])


def test_workspace_of_weights_is_bounded(sls):
    """A wide page table does not make a call of short sequences ask for gigabytes."""
    from paper_2607_19368_gb300 import small_cache as C
    for B, Hq, Hkv, hd, page, cols in [(256, 32, 8, 128, 64, 2048), (64, 12, 12, 64, 16, 8192),
                                       (4096, 128, 1, 128, 128, 1024), (1, 40, 8, 128, 1024, 2 ** 20),
                                       (65536, 128, 128, 64, 1024, 2 ** 20)]:
        for T in (B, 2 * B, 32 * B):
            size = C._bytes("weights", 0, 1, 0, (T, Hq, 1), (Hkv, hd, page, 1000, B, cols))
            assert 0 < size <= 2 ** 30 + 2 ** 24 + 8 * T * Hq, (B, Hq, cols, T)


@pytest.mark.parametrize("width", [1024, 131072])
def test_weights_of_single_tokens_behind_a_wide_table(sls, width):
    """The same sums whichever way the table's width sends the call."""
    B, Hq, Hkv, hd, page = 40, 64, 2, 64, 32
    m = [(37 * i) % 900 + 1 for i in range(B)]
    b = R.make_batch([1] * B, m, Hq, Hkv, hd, page, torch.float16, seed=52)
    table = torch.full((B, width // page), 1 << 29, dtype=torch.int32, device="cuda")
    table[:, :b["table"].shape[1]] = b["table"][:, :table.shape[1]]
    zero = torch.zeros(b["k"].shape[0], Hkv, page, device="cuda")
    want, bound = S.weights(b, zero)
    got = sls.attention_weights(b["q"], b["k"], table, b["kv_lens"], zero.clone())
    S.check(got, want, bound, "weights")


# ---------------------------------------------------------------------------
# layers
# ---------------------------------------------------------------------------

def test_layers_that_share_their_lengths(sls):
    """Each layer's cut takes a copy of the lengths before it; the lengths that are left are one."""
    m, page, Hkv, hd, keep = [90, 12, 300], 16, 2, 32, 40
    layers = [R.make_batch([1] * 3, m, Hkv, Hkv, hd, page, torch.float16, seed=7) for _ in range(3)]
    lens, table = layers[0]["kv_lens"], layers[0]["table"]
    after = None
    for i, b in enumerate(layers):
        g = torch.Generator("cpu").manual_seed(i)
        w = torch.rand(b["k"].shape[0], Hkv, page, generator=g)
        host = {k: (v.cpu() if torch.is_tensor(v) else v) for k, v in b.items()}
        want = S.evict(host, w, keep, 2, 8)
        w, after = w.cuda(), lens.clone()
        kept = sls.cache_evict(b["k"], b["v"], table, after, w, keep, first=2, last=8)
        assert torch.equal(kept.cpu(), want["kept"]) and torch.equal(w.cpu(), want["w"])
        assert torch.equal(b["k"].cpu().view(torch.int16), want["k"])
        assert after.tolist() == [40, 12, 40]
    # over lengths that are cut already a layer is left alone
    before = layers[0]["k"].clone()
    kept = sls.cache_evict(layers[0]["k"], layers[0]["v"], table, after, w, keep, first=2, last=8)
    assert torch.equal(layers[0]["k"].view(torch.int16), before.view(torch.int16))
    assert after.tolist() == [40, 12, 40] and kept[0, 0].tolist() == list(range(40))
