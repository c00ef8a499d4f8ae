"""Plain float64 statement of the attention calls, sequence by sequence, with
the bounds their float32 / 16-bit arithmetic stays within.  Inputs live on any
device; nothing of the package is used."""
import math

import torch

# unit roundoff of the 16-bit types
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# smallest half step of float16 (values below 2^-14 have absolute spacing 2^-24)
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def make_batch(new, m, Hq, Hkv, hd, page, dtype, seed, device="cuda", fill=float("nan"),
               spare_pages=3, q_scale=2.0, order="tokens"):
    """Packed queries and a cache whose every slot that no sequence covers holds
    `fill`.  new, m: lists of new tokens and cache lengths.  order: 'tokens' (slots
    outside heads) or 'heads' (heads outside slots)."""
    g = torch.Generator("cpu").manual_seed(seed)
    B, T = len(new), sum(new)
    pages = [max(0, -(-x // page)) for x in m]
    total = sum(pages) + spare_pages
    perm = torch.randperm(total, generator=g).tolist()
    width = max(pages + [1]) + 1
    table = torch.full((B, width), total + 1000, dtype=torch.int32)  # unused entries: no page
    shape = (total, page, Hkv, hd) if order == "tokens" else (total, Hkv, page, hd)
    k = torch.full(shape, fill, dtype=torch.float32)
    v = torch.full(shape, fill, dtype=torch.float32)
    if order == "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    at = 0
    for b in range(B):
        for p in range(pages[b]):
            table[b, p] = perm[at]
            used = min(page, m[b] - p * page)
            k[perm[at], :used] = torch.randn(used, Hkv, hd, generator=g)
            v[perm[at], :used] = torch.randn(used, Hkv, hd, generator=g)
            at += 1
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(new, dtype=torch.int32), 0)
    q = torch.randn(T, Hq, hd, generator=g) * q_scale

    def put(x):
        # .to keeps the strides of a dense permuted tensor
        return x.to(device=device, dtype=dtype)

    return {"q": put(q), "k": put(k), "v": put(v), "table": table.to(device),
            "kv_lens": torch.tensor(m, dtype=torch.int32, device=device), "cu": cu.to(device),
            "new": new, "m": m, "page": page}


def gather(cache, table_row, length, page):
    idx = torch.arange(length, device=cache.device)
    return cache[table_row[idx // page].long(), idx % page]


def attention(b, causal=True, scale=None):
    """(out, bound): float64 result per packed row and the largest distance that
    the kernels' arithmetic may put between theirs and it:
      rounding of the result                      u |o|
      rounding of the weights to 16 bits          u sum p |v|   (+ tiny sum |v| / l)
      float32 scores: products exact, hd sums     2^-23 hd scale |q|.|k| on s, as much
                                                  again relative on p, twice (p and sum)
      exp, the running sum, one division          2^-18 sum p |v|
    with p the softmax weights; a weight's exponent argument |s - max| up to a few
    hundred is rounded to float32, 2^-16 relative at most (inside the 2^-15 below)."""
    q, page = b["q"].double(), b["page"]
    T, Hq, hd = q.shape
    Hkv = b["k"].shape[2]
    dt = b["q"].dtype
    scale = hd ** -0.5 if scale is None else scale
    out = torch.zeros_like(q)
    bound = torch.zeros_like(q)
    t0 = 0
    for s, (n, m) in enumerate(zip(b["new"], b["m"])):
        if n and m:
            K = gather(b["k"], b["table"][s], m, page).double()
            V = gather(b["v"], b["table"][s], m, page).double()
            i = torch.arange(n, device=q.device)[:, None]
            j = torch.arange(m, device=q.device)[None, :]
            see = (j <= m - n + i) if causal else torch.ones(n, m, dtype=torch.bool,
                                                             device=q.device)
            some = see.any(-1)
            for h in range(Hq):
                c = h // (Hq // Hkv)
                Q, Kc, Vc = q[t0:t0 + n, h], K[:, c], V[:, c]
                S = (Q @ Kc.T * scale).masked_fill(~see, -math.inf)
                P = torch.softmax(S, -1).masked_fill(~see, 0.0)
                o = torch.where(some[:, None], P @ Vc, 0.0)
                A = P @ Vc.abs()
                d = (2.0 ** -23 * hd * scale * (Q.abs() @ Kc.abs().T)).masked_fill(~see, 0.0)
                d = d.amax(-1, keepdim=True) if m else d
                u = U[dt]
                top = S.amax(-1, keepdim=True)
                l = torch.exp(S - top).masked_fill(~see, 0.0).sum(-1, keepdim=True)
                spread = see.double() @ Vc.abs()
                err = u * o.abs() + (u + 2.0 ** -15 + 2 * d) * A + \
                    TINY[dt] * (1 + 2 * spread / l.clamp(min=1.0))
                out[t0:t0 + n, h] = o
                bound[t0:t0 + n, h] = torch.where(some[:, None], err, 0.0)
        t0 += n
    return out, bound


def append(q, k, v, b, positions, q_weight, k_weight, eps, inv_freq, interleaved, rope_scale,
           cu=True):
    """(q', cache k', cache v', bound of q', bound of k') in float64.  Bounds: one
    rounding to 16 bits, and 2^-19 of the terms of the rotation for the float32
    norm (sum of up to 128 squares, reciprocal root, two products), the cosine and
    sine (each to 2^-21) and the two products."""
    dt, page = b["k"].dtype, b["page"]
    K, V = b["k"].double().clone(), b["v"].double().clone()
    bK = torch.zeros_like(K)
    half = 0 if inv_freq is None else inv_freq.numel()

    def turn(x, w, pos):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        y, size = x.clone(), x.abs().clone()
        for i in range(half):
            a, c = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
            t = (pos.double() * inv_freq[i].double())[:, None]
            xa, xc = x[..., a], x[..., c]
            y[..., a] = rope_scale * (xa * torch.cos(t) - xc * torch.sin(t))
            y[..., c] = rope_scale * (xc * torch.cos(t) + xa * torch.sin(t))
            size[..., a] = size[..., c] = abs(rope_scale) * (xa.abs() + xc.abs())
        return y, U[dt] * y.abs() + 2.0 ** -19 * size + TINY[dt]

    qo, qb = torch.zeros_like(q, dtype=torch.float64), torch.zeros_like(q, dtype=torch.float64)
    t0 = 0
    for s, (n, m) in enumerate(zip(b["new"], b["m"])):
        idx = torch.arange(m - n, m, device=q.device)
        pos = positions[t0:t0 + n] if positions is not None else idx
        sl = slice(t0, t0 + n)
        qo[sl], qb[sl] = turn(q[sl], q_weight, pos)
        kk, kb = turn(k[sl], k_weight, pos)
        put = idx >= 0
        idx = idx.clamp(min=0)
        pg, st = b["table"][s][idx // page].long()[put], (idx % page)[put]
        K[pg, st], bK[pg, st], V[pg, st] = kk[put], kb[put], v[sl].double()[put]
        t0 += n
    return qo, K, V, qb, bK


def check(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() - bound
    worst = over.max().item() if over.numel() else 0.0
    assert worst <= 0.0, f"{what}: off by {worst:.3g} more than the bound"
