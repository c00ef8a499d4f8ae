"""Measured cases of the attention operators behind the compression pass: what
a model's attention layer does with the macro-tokens and their positions.

Three operators over one paged cache of keys and values:

* append: queries and keys normalised for each head (root mean square, a
  weight per element; optional) and rotated by their positions, the keys and
  values written to the cache;
* prefill: causal attention of packed prompts of different lengths over the
  cache, grouped heads, a history of earlier tokens allowed;
* decode: one query token per sequence over the cache.

A sequence s has n new tokens (cu_seqlens) and m tokens in the cache once they
are appended (kv_lens): new token i has cache index m - n + i and, under the
causal mask, sees the indices up to its own.  Index x of sequence s is slot
x % page_size of page page_table[s][x // page_size].

Head counts are those of the embedding widths of this repository's workloads at
128 elements a head (3584: 28, 4096: 32, 5120: 40) with 4 or 8 key heads, and
a few generic ones; lengths are those of its prompts after compression (512 / 4
to 131072 / 16) and, for decode, also of the uncompressed ones.
"""
import math

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one decode step's tokens of a few streams: latency counts
        {"name": "append 4 single tokens", "kind": "append", "dtype": "bf16", "Hq": 28, "Hkv": 4,
         "hd": 128, "B": 4, "n": 1, "hist": 2048, "page": 64, "norm": True, "rot": 128,
         "interleaved": False},
        # the macro-tokens of a batch of compressed prompts, ragged, halves rotated
        {"name": "append ragged prompts", "kind": "append", "dtype": "bf16", "Hq": 32, "Hkv": 8,
         "hd": 128, "B": 16, "n": 2048, "hist": 0, "page": 64, "norm": True, "rot": 128,
         "interleaved": False},
        # interleaved pairs, three quarters of a narrow head, short pages, no norm, fp16
        {"name": "append interleaved fp16", "kind": "append", "dtype": "fp16", "Hq": 25,
         "Hkv": 5, "hd": 64, "B": 7, "n": 1531, "hist": 300, "page": 16, "norm": False,
         "rot": 48, "interleaved": True},
        # a short prompt: 512 tokens at ratio 4, less than one tile of work for most of the GPU
        {"name": "prefill short prompt", "kind": "prefill", "dtype": "bf16", "Hq": 28, "Hkv": 4,
         "hd": 128, "B": 1, "n": 137, "hist": 0, "page": 64, "causal": True},
        # one 32k prompt at ratio 16
        {"name": "prefill one prompt", "kind": "prefill", "dtype": "bf16", "Hq": 28, "Hkv": 4,
         "hd": 128, "B": 1, "n": 2048, "hist": 0, "page": 64, "causal": True},
        # a ragged batch, pages that end inside a tile
        {"name": "prefill ragged batch", "kind": "prefill", "dtype": "bf16", "Hq": 32, "Hkv": 8,
         "hd": 128, "B": 8, "n": 2500, "hist": 0, "page": 16, "causal": True},
        # a further piece of a long prompt against what the cache holds already, fp16, narrow heads
        {"name": "prefill piece with history", "kind": "prefill", "dtype": "fp16", "Hq": 24,
         "Hkv": 8, "hd": 64, "B": 2, "n": 500, "hist": 7001, "page": 128, "causal": True},
        # a 131072-token prompt at ratio 16
        {"name": "prefill long prompt", "kind": "prefill", "dtype": "bf16", "Hq": 40, "Hkv": 8,
         "hd": 128, "B": 1, "n": 8192, "hist": 0, "page": 64, "causal": True},
        # a single stream behind a compressed prompt
        {"name": "decode one stream", "kind": "decode", "dtype": "bf16", "Hq": 28, "Hkv": 4,
         "hd": 128, "B": 1, "hist": 2061, "page": 64},
        # a serving batch of ragged lengths
        {"name": "decode ragged batch", "kind": "decode", "dtype": "bf16", "Hq": 32, "Hkv": 8,
         "hd": 128, "B": 64, "hist": 8192, "page": 16},
        # many short streams, narrow heads, as many key heads as query heads
        {"name": "decode many short fp16", "kind": "decode", "dtype": "fp16", "Hq": 12,
         "Hkv": 12, "hd": 64, "B": 200, "hist": 500, "page": 32},
        # a few uncompressed long prompts
        {"name": "decode long contexts", "kind": "decode", "dtype": "bf16", "Hq": 40, "Hkv": 8,
         "hd": 128, "B": 3, "hist": 131072, "page": 128},
    ]


HEADS = [(28, 4, 128), (32, 8, 128), (40, 8, 128), (24, 8, 64), (25, 5, 64), (12, 12, 64),
         (16, 1, 128), (14, 2, 80), (9, 3, 96)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    Hq, Hkv, hd = rng.choice(HEADS)
    case = {"kind": rng.choice(["append", "prefill", "prefill", "decode", "decode"]),
            "dtype": rng.choice(["bf16", "bf16", "fp16"]), "Hq": Hq, "Hkv": Hkv, "hd": hd,
            "page": rng.choice([16, 32, 64, 128])}
    if case["kind"] == "append":
        B = _log(rng, 1, 64)
        rot = hd if rng.random() < 0.6 else 16 * rng.randint(1, hd // 16)
        case.update(B=B, n=_log(rng, 1, max(2, 24000 // B)), hist=rng.randint(0, 3000),
                    norm=rng.random() < 0.6, rot=rot, interleaved=rng.random() < 0.5)
    elif case["kind"] == "prefill":
        # the largest listed case is 8192 tokens of 40 heads: padded pairs of all heads stay below
        B = _log(rng, 1, 12)
        cap = 40 * 8192 * 8192 // 2
        n = _log(rng, 1, math.isqrt(cap // (B * Hq)))
        room = cap // (B * Hq * n) - n
        hist = 0 if rng.random() < 0.5 or room < 1 else _log(rng, 1, min(16000, room))
        case.update(B=B, n=n, hist=hist, causal=rng.random() < 0.85)
    else:
        B = _log(rng, 1, 256)
        case.update(B=B, hist=_log(rng, 1, max(2, min(131072, 3 * 131072 * 8 * 128
                                                      // (2 * B * Hkv * hd)))))
    return case


def _lengths(case, gen):
    """(new tokens, cache lengths) of the sequences: the first is the longest, the
    others spread down from it."""
    B, n, hist = case["B"], case.get("n", 1), case["hist"]
    u = torch.rand(B, generator=gen)
    w = torch.rand(B, generator=gen)
    u[0] = w[0] = 1.0
    if case["kind"] == "decode":
        m = (1 + u * (hist - 1)).round().long()
        return torch.ones(B, dtype=torch.long), m.clamp(min=1)
    new = (n * (0.25 + 0.75 * u)).round().long().clamp(min=1)
    return new, new + (hist * w).round().long()


def _host(case):
    """What does not depend on the seed: the lengths of the sequences."""
    gen = torch.Generator().manual_seed(1234 + 7 * case["B"] + 31 * case["hist"])
    return _lengths(case, gen)


def prepare(case, seed):
    new, m = _host(case)
    B, T, ps = case["B"], int(new.sum()), case["page"]
    Hq, Hkv, hd, dt = case["Hq"], case["Hkv"], case["hd"], DT[case["dtype"]]
    g = torch.Generator(DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dt)

    width = -(-int(m.max()) // ps)
    pages = -(-m // ps)
    total = int(pages.sum())
    # every sequence's pages lie scattered over the cache, as an allocator leaves them
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    first = torch.cumsum(pages, 0) - pages
    cols = torch.arange(width)
    at = (first[:, None] + cols[None, :]).clamp(max=total - 1).to(DEV)
    table = torch.where((cols[None, :] < pages[:, None]).to(DEV), order[at], 0).contiguous()
    # keys of unit elements and queries that make scores of a few units' spread
    s = {"cache_k": normal(total, ps, Hkv, hd), "cache_v": normal(total, ps, Hkv, hd),
         "table": table, "kv_lens": m.to(torch.int32).to(DEV),
         "max_new": int(new.max()), "max_kv": int(m.max()), "page": ps,
         "kind": case["kind"], "causal": case.get("causal", True)}
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(new, 0)
    s["cu"] = cu.to(DEV)
    if case["kind"] == "append":
        # the three are slices of one projection's output
        qkv = normal(T, Hq + 2 * Hkv, hd)
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
            s["q_weight"] = (1 + 0.1 * normal(hd).float()).to(dt)
            s["k_weight"] = (1 + 0.1 * normal(hd).float()).to(dt)
        half = case["rot"] // 2
        s["inv_freq"] = (1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(DEV)
        s["interleaved"] = case["interleaved"]
    else:
        s["q"] = normal(T, Hq, hd, scale=2.0)
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
    ang = s["positions"].float()[:, None] * s["inv_freq"][None, :]
    c, n = ang.cos()[:, None, :], ang.sin()[:, None, :]
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = part[..., :half], part[..., half:]
        part = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([part, rest], -1)


def _plain_append(s):
    dt = s["q"].dtype
    seq, i = _token_rows(s)
    cu = s["cu"].long()
    idx = s["kv_lens"].long()[seq] - (cu[seq + 1] - cu[seq]) + i
    page = s["table"][seq, idx // s["page"]].long()
    slot = idx % s["page"]
    s["cache_k"][page, slot] = _rotate(s["k"], s["k_weight"], s).to(dt)
    s["cache_v"][page, slot] = s["v"]
    return {"q": _rotate(s["q"], s["q_weight"], s).to(dt), "k": s["cache_k"], "v": s["cache_v"]}


def _plain_attention(s):
    dt, hd = s["q"].dtype, s["q"].shape[-1]
    B, nmax, mmax = s["kv_lens"].shape[0], s["max_new"], s["max_kv"]
    Hkv = s["cache_k"].shape[2]
    G = s["q"].shape[1] // Hkv
    cu, m = s["cu"].long(), s["kv_lens"].long()
    n = cu[1:] - cu[:-1]
    j = torch.arange(mmax, device=DEV)
    i = torch.arange(nmax, device=DEV)
    page = s["table"].long()[:, j // s["page"]]
    slot = (j % s["page"]).expand(B, mmax)
    K = s["cache_k"][page, slot].float().permute(0, 2, 1, 3)             # B, Hkv, mmax, hd
    V = s["cache_v"][page, slot].float().permute(0, 2, 1, 3)
    rows = (cu[:-1, None] + i[None, :]).clamp(max=s["q"].shape[0] - 1)
    Q = s["q"][rows].float().view(B, nmax, Hkv, G, hd).permute(0, 2, 3, 1, 4)
    S = torch.matmul(Q.reshape(B, Hkv, G * nmax, hd), K.transpose(2, 3)).mul_(hd ** -0.5)
    S = S.view(B, Hkv, G, nmax, mmax)
    top = m[:, None].expand(B, nmax)
    if s["causal"]:
        top = (m - n)[:, None] + i[None, :] + 1
    hide = j[None, None, :] >= top[:, :, None]                           # B, nmax, mmax
    S.masked_fill_(hide[:, None, None], float("-inf"))
    P = torch.exp(S.sub_(S.amax(-1, keepdim=True)))
    O = torch.matmul(P.view(B, Hkv, G * nmax, mmax), V).view(B, Hkv, G, nmax, hd)
    O = O / P.sum(-1, keepdim=True)
    seq, at = _token_rows(s)
    return O.permute(0, 3, 1, 2, 4)[seq, at].reshape(s["q"].shape).to(dt)


def run(s):
    if not own:
        return _plain_append(s) if s["kind"] == "append" else _plain_attention(s)
    import paper_2607_19368_gb300 as sls
    if s["kind"] == "append":
        rope = s.get("rope")
        if rope is None:
            rope = s["rope"] = sls.Rope(s["inv_freq"], interleaved=s["interleaved"])
        q = sls.qkv_append(s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["table"],
                           s["kv_lens"], cu_seqlens=s["cu"], positions=s["positions"],
                           q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, rope=rope)
        return {"q": q, "k": s["cache_k"], "v": s["cache_v"]}
    if s["kind"] == "prefill":
        return sls.attention_prefill(s["q"], s["cache_k"], s["cache_v"], s["table"],
                                     s["kv_lens"], s["cu"], causal=s["causal"])
    return sls.attention_decode(s["q"], s["cache_k"], s["cache_v"], s["table"], s["kv_lens"])


def work(case):
    new, m = _host(case)
    Hq, Hkv, hd = case["Hq"], case["Hkv"], case["hd"]
    T = int(new.sum())
    if case["kind"] == "append":
        n = T * (Hq + 2 * Hkv) * hd
        return {"bytes": 2 * 2 * n + 4 * T, "flops": 10 * n}
    kv = 2 * 2 * Hkv * hd * int(m.sum())
    if case.get("causal", True):
        pairs = int((new * (m - new) + new * (new + 1) // 2).sum())
    else:
        pairs = int((new * m).sum())
    return {"bytes": kv + 2 * 2 * T * Hq * hd, "flops": 4 * hd * Hq * pairs}


# ---------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence and token by token
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


def exact(case, seed):
    s = prepare(case, seed)
    new, m = (x.tolist() for x in _host(case))
    ps, hd = case["page"], case["hd"]
    if case["kind"] != "append" and work(case)["flops"] > 4e12:
        return None
    if case["kind"] == "append":
        out = {"q": s["q"].double(), "k": s["cache_k"].double(), "v": s["cache_v"].double()}
    else:
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    t0 = 0
    for b, (n, length) in enumerate(zip(new, m)):
        t1 = t0 + n
        if case["kind"] == "append":
            where = torch.arange(length - n, length, device=DEV)
            page, slot = s["table"][b].long()[where // ps], where % ps
            pos = s["positions"][t0:t1]
            out["q"][t0:t1] = _exact_turn(s["q"][t0:t1], s["q_weight"], pos, s["inv_freq"],
                                          case["interleaved"])
            out["k"][page, slot] = _exact_turn(s["k"][t0:t1], s["k_weight"], pos, s["inv_freq"],
                                               case["interleaved"])
            out["v"][page, slot] = s["v"][t0:t1].double()
        else:
            used = s["table"][b, :-(-length // ps)].long()
            for h in range(case["Hq"]):
                c = h // (case["Hq"] // case["Hkv"])
                K = s["cache_k"][used, :, c].reshape(-1, hd)[:length].double()
                V = s["cache_v"][used, :, c].reshape(-1, hd)[:length].double()
                S = s["q"][t0:t1, h].double() @ K.T / math.sqrt(hd)
                if case.get("causal", True):
                    S += torch.full_like(S, -math.inf).triu(length - n + 1)
                out[t0:t1, h] = torch.softmax(S, -1) @ V
        t0 = t1
    return out
