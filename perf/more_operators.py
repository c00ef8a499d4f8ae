"""Measured cases of the operators that make the cache smaller: a cache of 8 bits with
the attention that reads it, and eviction by accumulated attention weight.

Five operators over one paged cache of keys and values (pages x page x key heads x head):

* append: queries and keys normalised for each head (optional) and rotated by their
  positions, keys and values written as 8-bit codes (e4m3 or int8) with a power-of-two
  scale for each block of tokens and key head;
* decode, prefill: softmax attention of one token per sequence, and of packed tokens,
  over such a cache;
* weights: the softmax weights that queries place on the cached tokens, summed over a key
  head's query heads and the queries, added to a running sum of every token and key head
  (16- or 8-bit keys);
* evict: of every sequence and key head the first and last tokens and the heaviest others
  are kept, in order, keys, values and weights moved to the front.

A sequence s has n new tokens (cu_seqlens) and m tokens in the cache (kv_lens): new token i
has cache index m - n + i and, under the causal mask, sees the indices up to its own.  Index
x of sequence s is slot x % page of page page_table[s][x // page]; its block is slot // block.

Head counts are those of the embedding widths of this repository's workloads at 128
elements a head (3584: 28, 4096: 32, 5120: 40) with 4 or 8 key heads, and a few generic
ones; lengths are those of its prompts, compressed (512 / 4 to 131072 / 16) or not.
"""
import math

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
# the largest code, and that as mantissa (in [0.5, 1)) and exponent
QMAX = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
MANT = {torch.int8: (0.9921875, 7), torch.float8_e4m3fn: (0.875, 9)}


def listed():
    return [
        # one decode step's tokens of a few streams: latency counts
        {"name": "append8 4 single tokens", "kind": "append", "dtype": "bf16", "code": "e4m3",
         "Hq": 28, "Hkv": 4, "hd": 128, "B": 4, "n": 1, "hist": 2048, "page": 64, "block": 64,
         "norm": True, "rot": 128, "interleaved": False},
        # the macro-tokens of a batch of compressed prompts, ragged, halves rotated
        {"name": "append8 ragged prompts", "kind": "append", "dtype": "bf16", "code": "e4m3",
         "Hq": 32, "Hkv": 8, "hd": 128, "B": 16, "n": 2048, "hist": 0, "page": 64, "block": 64,
         "norm": True, "rot": 128, "interleaved": False},
        # narrow heads behind a history that ends inside a block, int8, as it comes, short pages
        {"name": "append8 int8 with history", "kind": "append", "dtype": "fp16", "code": "int8",
         "Hq": 25, "Hkv": 5, "hd": 64, "B": 7, "n": 1531, "hist": 300, "page": 16, "block": 16,
         "norm": False, "rot": 0, "interleaved": False},
        # a single stream behind a compressed prompt: latency counts
        {"name": "decode8 one stream", "kind": "decode", "dtype": "bf16", "code": "e4m3",
         "Hq": 28, "Hkv": 4, "hd": 128, "B": 1, "hist": 2061, "page": 64, "block": 64},
        # a serving batch of ragged lengths
        {"name": "decode8 ragged batch", "kind": "decode", "dtype": "bf16", "code": "int8",
         "Hq": 32, "Hkv": 8, "hd": 128, "B": 64, "hist": 8192, "page": 16, "block": 16},
        # a few uncompressed long prompts
        {"name": "decode8 long contexts", "kind": "decode", "dtype": "fp16", "code": "e4m3",
         "Hq": 40, "Hkv": 8, "hd": 128, "B": 3, "hist": 131072, "page": 128, "block": 32},
        # a further piece of a long prompt against what the cache holds already, narrow heads
        {"name": "prefill8 piece with history", "kind": "prefill", "dtype": "fp16",
         "code": "int8", "Hq": 24, "Hkv": 8, "hd": 64, "B": 2, "n": 500, "hist": 7001,
         "page": 128, "block": 32, "causal": True},
        # a 131072-token prompt at ratio 16
        {"name": "prefill8 long prompt", "kind": "prefill", "dtype": "bf16", "code": "e4m3",
         "Hq": 40, "Hkv": 8, "hd": 128, "B": 1, "n": 8192, "hist": 0, "page": 64, "block": 64,
         "causal": True},
        # the weights of a decode step's tokens, summed from step to step, 16-bit keys
        {"name": "weights decode batch", "kind": "weights", "dtype": "bf16", "code": "16",
         "Hq": 32, "Hkv": 8, "hd": 128, "B": 32, "n": 1, "hist": 4096, "page": 64, "block": 64},
        # the last 32 tokens of a long prompt vote on what is kept of it
        {"name": "weights window of a prompt", "kind": "weights", "dtype": "bf16",
         "code": "e4m3", "Hq": 28, "Hkv": 4, "hd": 128, "B": 1, "n": 32, "hist": 32768,
         "page": 64, "block": 64},
        # a long prompt's cache cut to a sixteenth, 16 bits
        {"name": "evict one prompt", "kind": "evict", "dtype": "bf16", "code": "16",
         "Hq": 28, "Hkv": 4, "hd": 128, "B": 1, "hist": 32768, "keep": 2048, "first": 4,
         "last": 32, "page": 64, "block": 64},
        # a ragged batch cut to a common budget, 8 bits; some sequences are below it
        {"name": "evict ragged batch", "kind": "evict", "dtype": "bf16", "code": "e4m3",
         "Hq": 32, "Hkv": 8, "hd": 128, "B": 24, "hist": 8192, "keep": 1024, "first": 4,
         "last": 64, "page": 64, "block": 16},
    ]


HEADS = [(28, 4, 128), (32, 8, 128), (40, 8, 128), (24, 8, 64), (25, 5, 64), (12, 12, 64),
         (16, 1, 128), (14, 2, 80), (9, 3, 96)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    Hq, Hkv, hd = rng.choice(HEADS)
    kind = rng.choice(["append", "decode", "decode", "prefill", "weights", "evict"])
    page = rng.choice([16, 32, 64, 128])
    case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "fp16"]),
            "code": rng.choice(["e4m3", "int8"]), "Hq": Hq, "Hkv": Hkv, "hd": hd,
            "page": page, "block": rng.choice([b for b in (16, 32, 64, 128) if b <= page])}
    if kind in ("weights", "evict"):
        case["code"] = rng.choice(["16", "16", "e4m3", "int8"])
    if kind == "append":
        B = _log(rng, 1, 64)
        # int8 codes are whole numbers, the same on both sides only where nothing rounds first
        turn = case["code"] == "e4m3"
        rot = 0 if not turn else hd if rng.random() < 0.6 else 16 * rng.randint(1, hd // 16)
        case.update(B=B, n=_log(rng, 1, max(2, 24000 // B)), hist=rng.randint(0, 3000),
                    norm=turn and rng.random() < 0.6, rot=rot, interleaved=rng.random() < 0.5)
    elif kind == "prefill":
        # the largest listed case is 8192 tokens of 40 heads: padded pairs of all heads stay below
        B = _log(rng, 1, 12)
        cap = 40 * 8192 * 8192 // 2
        n = _log(rng, 1, math.isqrt(cap // (B * Hq)))
        room = cap // (B * Hq * n) - n
        hist = 0 if rng.random() < 0.5 or room < 1 else _log(rng, 1, min(16000, room))
        case.update(B=B, n=n, hist=hist, causal=rng.random() < 0.85)
    elif kind == "decode":
        B = _log(rng, 1, 256)
        case.update(B=B, hist=_log(rng, 1, max(2, min(131072, 3 * 131072 * 8 * 128
                                                      // (2 * B * Hkv * hd)))))
    elif kind == "weights":
        # up to four times the listed window's scores, tokens with all of their heads
        B = _log(rng, 1, 64)
        n = 1 if rng.random() < 0.4 else _log(rng, 2, 64)
        most = min(131072, 4 * 28 * 32 * 32768 // (B * Hq * n), (1 << 28) // (B * Hkv * hd))
        case.update(B=B, n=n, hist=_log(rng, 1, max(2, most)))
    else:
        B = _log(rng, 1, 64)
        hist = _log(rng, 16, max(17, min(131072, (1 << 28) // (B * Hkv * hd))))
        keep = _log(rng, 1, hist)
        first = rng.randint(0, min(8, keep // 2))
        case.update(B=B, hist=hist, keep=keep, first=first,
                    last=rng.randint(0, min(128, keep - first)))
    return case


def _host(case):
    """What does not depend on the seed: new tokens and cache lengths of the sequences; the
    first is the longest, the others spread down from it."""
    gen = torch.Generator().manual_seed(1234 + 7 * case["B"] + 31 * case["hist"])
    B, n, hist = case["B"], case.get("n", 1), case["hist"]
    u = torch.rand(B, generator=gen)
    w = torch.rand(B, generator=gen)
    u[0] = w[0] = 1.0
    if case["kind"] in ("decode", "evict"):
        m = (1 + u * (hist - 1)).round().long()
        return torch.ones(B, dtype=torch.long), m.clamp(min=1)
    if case["kind"] == "weights":
        m = n + (hist * w).round().long()
        return torch.full((B,), n, dtype=torch.long), m
    new = (n * (0.25 + 0.75 * u)).round().long().clamp(min=1)
    return new, new + (hist * w).round().long()


def _scale_of(a, code):
    """The least power of two s >= 2^-126 with a <= the largest code times s."""
    top, e = MANT[code]
    mant, exp = torch.frexp(a)
    exp = torch.where(a > 0, exp - e + (mant > top).int(), -126).clamp(min=-126).int()
    return ((exp + 127) << 23).view(torch.float32)     # ldexp goes by pow, which may round


def _to_code(x, code):
    """Values in units of the scale, rounded to codes."""
    q = QMAX[code]
    x = x.clamp(-q, q)
    return x.round().to(code) if code == torch.int8 else x.to(code)


def _bytes(t):
    return t.view(torch.uint8)


def prepare(case, seed):
    new, m = _host(case)
    B, T, ps, blk = case["B"], int(new.sum()), case["page"], case["block"]
    Hq, Hkv, hd, dt = case["Hq"], case["Hkv"], case["hd"], DT[case["dtype"]]
    g = torch.Generator(DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale)

    width = -(-int(m.max()) // ps)
    pages = -(-m // ps)
    total = int(pages.sum())
    # every sequence's pages lie scattered over the cache, as an allocator leaves them
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    first = torch.cumsum(pages, 0) - pages
    cols = torch.arange(width)
    at = (first[:, None] + cols[None, :]).clamp(max=total - 1).to(DEV)
    table = torch.where((cols[None, :] < pages[:, None]).to(DEV), order[at], 0).contiguous()
    s = {"table": table, "kv_lens": m.to(torch.int32).to(DEV), "kind": case["kind"],
         "max_new": int(new.max()), "max_kv": int(m.max()), "page": ps, "block": blk,
         "causal": case.get("causal", True), "k_scale": None, "v_scale": None}
    for x in "kv":
        # unit elements, tokens of different size
        c = normal(total, ps, Hkv, hd)
        c.mul_(torch.exp(normal(total, ps, Hkv, 1, scale=0.25)))
        if case["code"] == "16":
            s["cache_" + x] = c.to(dt)
        else:
            code = CODE[case["code"]]
            c = c.view(total, ps // blk, blk, Hkv, hd)
            sc = _scale_of(c.abs().amax((2, 4)), code)
            s["cache_" + x] = _to_code(c / sc[:, :, None, :, None], code).view(total, ps, Hkv, hd)
            s[x + "_scale"] = sc
        del c
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(new, 0)
    s["cu"] = cu.to(DEV)
    if case["kind"] == "append":
        # the three are slices of one projection's output
        qkv = normal(T, Hq + 2 * Hkv, hd)
        qkv = qkv.mul_(torch.exp(normal(T, 1, 1, scale=0.25))).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        # macro-tokens' positions: rising, with gaps of up to 2 * 16
        step = torch.randint(1, 32, (T,), generator=g, device=DEV)
        rise = torch.cumsum(step, 0)
        base = torch.repeat_interleave(torch.arange(B), new).to(DEV)
        off = rise[s["cu"][:-1].long()] - step[s["cu"][:-1].long()]
        hist = 16 * (m - new).to(DEV)
        s["positions"] = (rise - off[base] + hist[base]).to(torch.int32)
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"] = (1 + 0.1 * normal(hd)).to(dt)
            s["k_weight"] = (1 + 0.1 * normal(hd)).to(dt)
        half = case["rot"] // 2
        s["inv_freq"] = (1e6 ** (-torch.arange(half, dtype=torch.float64) / max(1, half)))
        s["inv_freq"] = s["inv_freq"].float().to(DEV)
        s["interleaved"] = case["interleaved"]
    elif case["kind"] == "evict":
        # a few tokens carry much of the weight
        w = torch.exp(normal(total, Hkv, ps, scale=2.0)) * 1e-2
        s.update(weights0=w, weights=w.clone(), lens0=s["kv_lens"].clone(), keep=case["keep"],
                 first=case["first"], last=case["last"])
    else:
        # scores of a unit's or two's spread
        s["q"] = normal(T, Hq, hd, scale=1.5).to(dt)
        if case["kind"] == "weights":
            # a decode step adds to the sum of the steps before it; a window starts it
            s["weights"] = torch.zeros(total, Hkv, ps, device=DEV)
            if case["n"] == 1:
                part = torch.exp(normal(total, Hkv, ps)) * (64.0 * Hq / Hkv / s["max_kv"])
                s["weights"].copy_(part)
    return s


# ---------------------------------------------------------------------------
# plain forms: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------

def _token_rows(s):
    """For every packed token: its sequence and its place among the new ones."""
    t = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return seq, t - s["cu"].long()[seq]


def _rotate(x, weight, s):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
    half = s["inv_freq"].numel()
    ang = s["positions"].double()[:, None] * s["inv_freq"].double()[None, :]
    c, n = ang.cos().float()[:, None, :], ang.sin().float()[:, None, :]
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = part[..., :half], part[..., half:]
        part = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([part, rest], -1)


def _put_codes(y, cache, scale, s, place):
    """New values y (T x heads x elements) into the cache's codes and scales."""
    seq, idx, page, slot, before = place
    code, blk = cache.dtype, s["block"]
    per = s["page"] // blk
    flat = page * per + slot // blk                                       # block of every token
    table = scale.view(-1, scale.shape[-1])
    most = torch.zeros_like(table)
    most = most.scatter_reduce(0, flat[:, None].expand(-1, y.shape[1]), y.abs().amax(-1), "amax")
    fresh = _scale_of(most, code)
    # the one block of a sequence that holds earlier tokens as well as new ones
    B = before.shape[0]
    start = before // blk * blk
    col = (before // s["page"]).clamp(max=s["table"].shape[1] - 1)
    held = s["table"][torch.arange(B, device=DEV), col].long()
    part = held * per + before % s["page"] // blk
    old = table[part]
    now = torch.where((before > start)[:, None], torch.maximum(fresh[part], old), fresh[part])
    fresh[part] = now
    i = torch.arange(blk, device=DEV)
    at = (start % s["page"])[:, None] + i[None, :]
    bytes_ = _bytes(cache)
    was = bytes_[held[:, None], at]
    again = _to_code(was.view(code).float() * (old / now)[:, None, :, None], code)
    keep = (i[None, :] < (before - start)[:, None])[..., None, None]
    bytes_[held[:, None], at] = torch.where(keep, _bytes(again), was)
    table[flat] = fresh[flat]
    bytes_[page, slot] = _bytes(_to_code(y / fresh[flat][..., None], code))


def _plain_append(s):
    dt = s["q"].dtype
    seq, i = _token_rows(s)
    cu = s["cu"].long()
    before = s["kv_lens"].long() - (cu[1:] - cu[:-1])
    idx = before[seq] + i
    page = s["table"][seq, idx // s["page"]].long()
    place = (seq, idx, page, idx % s["page"], before)
    _put_codes(_rotate(s["k"], s["k_weight"], s), s["cache_k"], s["k_scale"], s, place)
    _put_codes(s["v"].float(), s["cache_v"], s["v_scale"], s, place)
    return {"q": _rotate(s["q"], s["q_weight"], s).to(dt), "k": s["cache_k"], "v": s["cache_v"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _gather(s, x):
    """The values of all sequences' cached tokens: B, heads, longest, elements."""
    cache, scale = s["cache_" + x], s[x + "_scale"]
    j = torch.arange(s["max_kv"], device=DEV)
    page = s["table"].long()[:, j // s["page"]]
    slot = (j % s["page"]).expand(page.shape)
    if scale is None:
        return cache[page, slot].float().permute(0, 2, 1, 3)
    c = _bytes(cache)[page, slot].view(cache.dtype).float()
    return (c * scale[page, slot // s["block"]][..., None]).permute(0, 2, 1, 3)


def _softmax(s):
    """Weights of all sequences' new rows: B, key heads, query heads of one, rows, keys; zero
    where a row is padding."""
    hd = s["q"].shape[-1]
    B, nmax, mmax = s["kv_lens"].shape[0], s["max_new"], s["max_kv"]
    K = _gather(s, "k")
    Hkv = K.shape[1]
    G = s["q"].shape[1] // Hkv
    cu, m = s["cu"].long(), s["kv_lens"].long()
    n = cu[1:] - cu[:-1]
    j = torch.arange(mmax, device=DEV)
    i = torch.arange(nmax, device=DEV)
    rows = (cu[:-1, None] + i[None, :]).clamp(max=s["q"].shape[0] - 1)
    Q = s["q"][rows].float().view(B, nmax, Hkv, G, hd).permute(0, 2, 3, 1, 4)
    S = torch.matmul(Q.reshape(B, Hkv, G * nmax, hd), K.transpose(2, 3)).mul_(hd ** -0.5)
    del K
    S = S.view(B, Hkv, G, nmax, mmax)
    top = m[:, None].expand(B, nmax)
    if s["causal"]:
        top = (m - n)[:, None] + i[None, :] + 1
    hide = j[None, None, :] >= top[:, :, None]                           # B, nmax, mmax
    S.masked_fill_(hide[:, None, None], float("-inf"))
    P = S.sub_(S.amax(-1, keepdim=True)).exp_()
    return P, P.sum(-1, keepdim=True)


def _plain_attention(s):
    P, l = _softmax(s)
    B, Hkv, G, nmax, mmax = P.shape
    V = _gather(s, "v")
    O = torch.matmul(P.view(B, Hkv, G * nmax, mmax), V).view(B, Hkv, G, nmax, -1) / l
    seq, at = _token_rows(s)
    return O.permute(0, 3, 1, 2, 4)[seq, at].reshape(s["q"].shape).to(s["q"].dtype)


def _plain_weights(s):
    P, l = _softmax(s)
    add = P.div_(l).sum((2, 3))                                           # B, Hkv, mmax
    B, Hkv, mmax = add.shape
    j = torch.arange(mmax, device=DEV)
    page = s["table"].long()[:, j // s["page"]]
    used = j[None, :] < s["kv_lens"].long()[:, None]
    b, x = used.nonzero(as_tuple=True)
    s["weights"][page[b, x], :, x % s["page"]] += add[b, :, x]
    return s["weights"]


def _plain_evict(s):
    s["kv_lens"].copy_(s["lens0"])
    s["weights"].copy_(s["weights0"])
    m, keep, ps, blk = s["kv_lens"].long(), s["keep"], s["page"], s["block"]
    B, mmax = m.shape[0], s["max_kv"]
    Hkv = s["weights"].shape[1]
    j = torch.arange(mmax, device=DEV)
    page = s["table"].long()[:, j // ps]
    slot = (j % ps).expand(B, mmax)
    w = s["weights"][page, :, slot].permute(0, 2, 1)                      # B, Hkv, mmax
    must = (j[None] < s["first"]) | ((j[None] >= (m - s["last"])[:, None]) & (j[None] < m[:, None]))
    rank = torch.where(must[:, None], torch.inf, w)
    rank = torch.where((j[None] < m[:, None])[:, None], rank, -torch.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    count = torch.minimum(m, torch.tensor(keep, device=DEV))
    best = torch.where(j[None, None, :best.shape[-1]] < count[:, None, None], best, 1 << 30)
    best = best.sort(-1).values                                           # in order
    real = best < (1 << 30)
    kept = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device=DEV)
    kept[..., :best.shape[-1]] = torch.where(real, best, -1).int()
    # rows that go to the front: (sequence, head, place) and where they come from
    b, h, to = (real & (count < m)[:, None, None]).nonzero(as_tuple=True)
    src = best[b, h, to]
    p0, s0 = page[b, src], src % ps
    p1, s1 = page[b, to], to % ps
    moved = s["weights"][p0, h, s0]
    over = (j[None] < m[:, None]) & (j[None] >= keep)
    bz, jz = over.nonzero(as_tuple=True)
    s["weights"][page[bz, jz], :, slot[bz, jz]] = 0.0
    s["weights"][p1, h, s1] = moved
    for x in "kv":
        cache, scale = s["cache_" + x], s[x + "_scale"]
        if scale is None:
            cache[p1, s1, h] = cache[p0, s0, h]
            continue
        code = cache.dtype
        rows = _bytes(cache)[p0, s0, h].view(code).float()
        was = scale[p0, s0 // blk, h]
        most = torch.zeros(scale.numel(), device=DEV)
        into = (p1 * (ps // blk) + s1 // blk) * Hkv + h
        most = most.scatter_reduce(0, into, was, "amax")
        rows = _to_code(rows * (was / most[into])[:, None], code)
        _bytes(cache)[p1, s1, h] = _bytes(rows)
        scale.view(-1)[into] = most[into]
    s["kv_lens"].copy_(count)
    return _evicted(s, kept)


def _evicted(s, kept):
    out = {"kept": kept, "k": s["cache_k"], "v": s["cache_v"], "weights": s["weights"],
           "kv_lens": s["kv_lens"]}
    if s["k_scale"] is not None:
        out.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return out


def run(s):
    kind = s["kind"]
    if not own:
        return {"append": _plain_append, "decode": _plain_attention, "prefill": _plain_attention,
                "weights": _plain_weights, "evict": _plain_evict}[kind](s)
    import paper_2607_19368_gb300 as sls
    if kind == "append":
        rope = s.get("rope")
        if rope is None and s["inv_freq"].numel():
            rope = s["rope"] = sls.Rope(s["inv_freq"], interleaved=s["interleaved"])
        q = sls.qkv_append_q8(s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["k_scale"],
                              s["v_scale"], s["table"], s["kv_lens"], cu_seqlens=s["cu"],
                              positions=s["positions"], q_weight=s["q_weight"],
                              k_weight=s["k_weight"], eps=1e-6, rope=rope)
        return {"q": q, "k": s["cache_k"], "v": s["cache_v"], "k_scale": s["k_scale"],
                "v_scale": s["v_scale"]}
    if kind == "decode":
        return sls.attention_decode_q8(s["q"], s["cache_k"], s["cache_v"], s["k_scale"],
                                       s["v_scale"], s["table"], s["kv_lens"])
    if kind == "prefill":
        return sls.attention_prefill_q8(s["q"], s["cache_k"], s["cache_v"], s["k_scale"],
                                        s["v_scale"], s["table"], s["kv_lens"], s["cu"],
                                        causal=s["causal"])
    if kind == "weights":
        return sls.attention_weights(s["q"], s["cache_k"], s["table"], s["kv_lens"],
                                     s["weights"], cu_seqlens=s["cu"], k_scale=s["k_scale"])
    # the sequences as they were before: a call shortens them
    s["kv_lens"].copy_(s["lens0"])
    s["weights"].copy_(s["weights0"])
    kept = sls.cache_evict(s["cache_k"], s["cache_v"], s["table"], s["kv_lens"], s["weights"],
                           s["keep"], first=s["first"], last=s["last"], k_scale=s["k_scale"],
                           v_scale=s["v_scale"])
    return _evicted(s, kept)


def work(case):
    new, m = _host(case)
    Hq, Hkv, hd, blk = case["Hq"], case["Hkv"], case["hd"], case["block"]
    T, total = int(new.sum()), int(m.sum())
    size = 2 if case["code"] == "16" else 1
    scales = 0 if size == 2 else 4 * Hkv * int((-(-m // blk)).sum())
    if case["causal"] if "causal" in case else True:
        pairs = int((new * (m - new) + new * (new + 1) // 2).sum())
    else:
        pairs = int((new * m).sum())
    if case["kind"] == "append":
        n = T * (Hq + 2 * Hkv) * hd
        blocks = int((-(-m // blk) - (m - new) // blk).sum())
        return {"bytes": 2 * n + 2 * T * Hq * hd + 2 * T * Hkv * hd + 8 * Hkv * blocks + 4 * T,
                "flops": 10 * n}
    if case["kind"] == "weights":
        return {"bytes": size * Hkv * hd * total + scales + 8 * Hkv * total + 2 * T * Hq * hd,
                "flops": 2 * hd * Hq * pairs}
    if case["kind"] == "evict":
        cut = m > case["keep"]
        moved = int(cut.sum()) * max(0, case["keep"] - case["first"])
        weights = 4 * Hkv * int((2 * m[cut]).sum())
        return {"bytes": 4 * size * Hkv * hd * moved + weights + 4 * Hkv * case["B"] * case["keep"]
                + (0 if size == 2 else 4 * 4 * Hkv * moved // blk),
                "flops": Hkv * total}
    return {"bytes": 2 * Hkv * hd * total + 2 * scales + 2 * 2 * T * Hq * hd,
            "flops": 4 * hd * Hq * pairs}


# ---------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence and head by head
# ---------------------------------------------------------------------------

def _exact_turn(x, weight, pos, inv_freq, interleaved):
    """One sequence's heads (n, H, hd), rotated as complex numbers."""
    x = x.double()
    if weight is not None:
        x = weight.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6)
    half = inv_freq.numel()
    turn = torch.polar(torch.ones(1, 1, dtype=torch.float64, device=DEV),
                       pos.double()[:, None] * inv_freq.double()[None, :])[:, None, :]
    out = x.clone()
    even = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    odd = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    z = torch.complex(x[..., even], x[..., odd]) * turn
    out[..., even], out[..., odd] = z.real, z.imag
    return out


def _exact_power(a, code):
    """The least power of two with a <= the largest code times it."""
    mant, exp = torch.frexp(a / QMAX[code])             # a / 448 = 2^-7 is exact, its log2 is not
    exp = torch.where(mant > 0.5, exp, exp - 1)
    exp = torch.where(a > 0, exp, -126).clamp(min=-126).long()
    return ((exp + 1023) << 52).view(torch.float64)


def _exact_blocks(s, case, b, cache, scale, y, codes, scales):
    """One sequence's new values y (n, heads, elements) of one of the two caches, block by
    block: what the codes stand for in units of the scale, before their rounding."""
    ps, blk, code = case["page"], case["block"], cache.dtype
    length = int(s["kv_lens"][b])
    n = y.shape[0]
    old = length - n
    for start in range(old // blk * blk, length, blk):
        page = int(s["table"][b, start // ps])
        at = start % ps
        lo, hi = max(start, old), min(start + blk, length)
        part = y[lo - old:hi - old]
        now = _exact_power(part.abs().amax((0, 2)), code)
        if start < old:
            was = scale[page, at // blk].double()
            now = torch.maximum(now, was)
            held = slice(at, at + old - start)
            codes[page, held] = cache[page, held].double() * (was / now)[:, None]
        scales[page, at // blk] = now
        codes[page, at + lo - start:at + hi - start] = part / now[:, None]


def exact(case, seed):
    if case["kind"] == "prefill" and work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    new, m = (x.tolist() for x in _host(case))
    ps, hd, blk, kind = case["page"], case["hd"], case["block"], case["kind"]
    G = case["Hq"] // case["Hkv"]
    if kind == "append":
        if sum(new) // blk + case["B"] > 3000:
            return None
        out = {"q": torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)}
        for x in "kv":
            out[x], out[x + "_scale"] = s["cache_" + x].double(), s[x + "_scale"].double()
        t0 = 0
        for b, n in enumerate(new):
            t1 = t0 + n
            f = s["inv_freq"], case["interleaved"]
            pos = s["positions"][t0:t1]
            out["q"][t0:t1] = _exact_turn(s["q"][t0:t1], s["q_weight"], pos, *f)
            k = _exact_turn(s["k"][t0:t1], s["k_weight"], pos, *f)
            for x, y in (("k", k), ("v", s["v"][t0:t1].double())):
                _exact_blocks(s, case, b, s["cache_" + x], s[x + "_scale"], y, out[x],
                              out[x + "_scale"])
            t0 = t1
        return out
    if kind == "evict":
        return _exact_evict(case, s, m)
    if kind == "weights":
        out = s["weights"].double()
    else:
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    if case["B"] * case["Hq"] > 4000:
        return None

    def values(x, used, c, length):
        v = s["cache_" + x][used, :, c].double()
        if s[x + "_scale"] is not None:
            v = v * s[x + "_scale"][used, :, c].double().repeat_interleave(blk, 1)[..., None]
        return v.reshape(-1, hd)[:length]

    t0 = 0
    for b, (n, length) in enumerate(zip(new, m)):
        t1 = t0 + n
        used = s["table"][b, :-(-length // ps)].long()
        where = torch.arange(length, device=DEV)
        page, slot = used[where // ps], where % ps
        for c in range(case["Hkv"]):
            K = values("k", used, c, length)
            V = None if kind == "weights" else values("v", used, c, length)
            for h in range(c * G, (c + 1) * G):
                S = s["q"][t0:t1, h].double() @ K.T / math.sqrt(hd)
                if case.get("causal", True):
                    S += torch.full_like(S, -math.inf).triu(length - n + 1)
                P = torch.softmax(S, -1)
                if kind == "weights":
                    out[page, c, slot] += P.sum(0)
                else:
                    out[t0:t1, h] = P @ V
        t0 = t1
    return out


def _exact_evict(case, s, m):
    """Sequence by sequence and head by head, on copies; codes as their values."""
    ps, blk, keep = case["page"], case["block"], case["keep"]
    if case["B"] * case["Hkv"] > 1600:
        return None
    kept = torch.full((case["B"], case["Hkv"], keep), -1, dtype=torch.int32, device=DEV)
    out = {"kept": kept, "k": s["cache_k"].double(), "v": s["cache_v"].double(),
           "weights": s["weights0"].double(), "kv_lens": s["lens0"].clone().clamp(max=keep)}
    eight = s["k_scale"] is not None
    if eight:
        out.update(k_scale=s["k_scale"].double(), v_scale=s["v_scale"].double())
    for b, length in enumerate(m):
        j = torch.arange(length, device=DEV)
        page, slot = s["table"][b].long()[j // ps], j % ps
        for h in range(case["Hkv"]):
            if length <= keep:
                kept[b, h, :length] = j.int()
                continue
            w = s["weights0"][page, h, slot].double()
            inner = w[case["first"]:length - case["last"]]
            some = torch.argsort(inner, descending=True, stable=True)
            some = some[:keep - case["first"] - case["last"]] + case["first"]
            idx = torch.cat([j[:case["first"]], some.sort().values, j[length - case["last"]:]])
            kept[b, h] = idx.int()
            to = (page[:keep], slot[:keep])
            out["weights"][page[keep:], h, slot[keep:]] = 0.0
            out["weights"][to[0], h, to[1]] = w[idx]
            for x in "kv":
                rows = s["cache_" + x][page[idx], slot[idx], h].double()
                if eight:
                    was = s[x + "_scale"][page[idx], slot[idx] // blk, h].double()
                    pad = torch.nn.functional.pad(was, (0, -keep % blk)).view(-1, blk)
                    now = pad.amax(-1)
                    rows = rows * (was / now.repeat_interleave(blk)[:keep])[:, None]
                    at = j[:keep:blk]
                    out[x + "_scale"][page[at], slot[at] // blk, h] = now
                out[x][to[0], to[1], h] = rows
    return out
