"""Plain float64 statements of the calls that make the cache smaller, sequence by sequence,
with the bounds that their arithmetic stays within.  Nothing of the package is used."""
import math

import torch

from tests import attention_ref as R

MOST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def power(a, code):
    """The least power of two s >= 2^-126 with a <= MOST s."""
    mant, exp = torch.frexp(a.double() / MOST[code])
    exp = torch.where(mant > 0.5, exp, exp - 1)
    exp = torch.where(a > 0, exp, -126).clamp(min=-126).long()
    return ((exp + 1023) << 52).view(torch.float64)  # ldexp goes by pow, which may round


def to_codes(x, code):
    x = x.clamp(-MOST[code], MOST[code])
    return x.round().to(code) if code == torch.int8 else x.float().to(code)


def half_step(x, code):
    """The largest distance of a number from its code, in units of the scale."""
    if code == torch.int8:
        return torch.full_like(x, 0.5)
    return torch.maximum(x.abs() * 2.0 ** -4, torch.full_like(x, 2.0 ** -10))


def index8(t, *at):
    """t[at] for types that indexing may not take."""
    return t.view(torch.uint8)[at].view(t.dtype)


def codes_of(b, code, block, spread=0.5, seed=0):
    """Replaces b's cache (make_batch) by codes of it and their scales; slots that no sequence
    covers hold NaN (or -128), and so do the scales of blocks without a covered slot."""
    g = torch.Generator("cpu").manual_seed(seed)
    out = dict(b, block=block)
    n, page, H, hd = b["k"].shape
    for x in "kv":
        c = b[x].double().cpu()
        hole = torch.isnan(c)
        c = c * torch.exp(spread * torch.randn(n, page, H, 1, generator=g)).double()
        c = c.masked_fill(hole, 0.0).view(n, page // block, block, H, hd)
        s = power(c.abs().amax((2, 4)), code)
        q = to_codes(c / s[:, :, None, :, None], code).view(n, page, H, hd)
        hole = hole.view(n, page, H, hd)
        q.view(torch.uint8)[hole] = 0x80 if code == torch.int8 else 0x7f
        used = (~hole).view(n, page // block, block, H, hd).any(4).any(2)
        s = torch.where(used, s, math.nan)
        dev = b[x].device
        out[x], out[x + "_scale"] = q.to(dev), s.float().to(dev)
    return out


def values(b, x):
    """The cache's values in float64; holes as NaN."""
    c, s = b[x], b[x + "_scale"]
    v = c.to(torch.float32).double()
    if c.dtype == torch.int8:
        v = torch.where(c == -128, math.nan, v)
    return v * s.double().repeat_interleave(b["block"], 1)[..., None]


def plain(b):
    """The batch with its cache as 64-bit values."""
    return dict(b, k=values(b, "k"), v=values(b, "v"))


def turned(x, w, eps, inv_freq, inter, rope_scale, pos):
    """(y, bound): normed and rotated rows in float64 and the distance float32 may add."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    y, size = x.clone(), x.abs().clone()
    half = 0 if inv_freq is None else inv_freq.numel()
    for i in range(half):
        a, c = (2 * i, 2 * i + 1) if inter else (i, half + i)
        t = (pos.double() * inv_freq[i].double())[:, None]
        xa, xc = x[..., a], x[..., c]
        y[..., a] = rope_scale * (xa * torch.cos(t) - xc * torch.sin(t))
        y[..., c] = rope_scale * (xc * torch.cos(t) + xa * torch.sin(t))
        size[..., a] = size[..., c] = abs(rope_scale) * (xa.abs() + xc.abs())
    # as in attention_ref.append: norm, turn and products in float32
    return y, (2.0 ** -19 * size if half or w is not None else 0.0 * size)


def append(b, x, y, err):
    """(values, bound, scales) of cache x after y (T x H x hd, error bound err) is appended:
    float64 value of every slot, the largest distance of code * scale from it."""
    code, block, page = b[x].dtype, b["block"], b["page"]
    V, S = values(b, x).clone(), b[x + "_scale"].double().clone()
    E = torch.zeros_like(V)
    t0 = 0
    for s, (n, m) in enumerate(zip(b["new"], b["m"])):
        old = max(0, m - n)
        cap = b["table"].shape[1] * page
        for start in range(old // block * block, min(m, cap), block):
            pg, at = int(b["table"][s, start // page]), start % page
            if not 0 <= pg < V.shape[0]:
                continue
            lo, hi = max(start, old), min(start + block, m, cap)
            if lo >= hi:
                continue
            r = slice(t0 + lo - (m - n), t0 + hi - (m - n))
            part = y[r]
            fin = torch.where(part.isfinite(), part.abs(), 0.0)
            now = power(fin.amax((0, 2)), code)
            if start < old:
                was = S[pg, at // block]
                now = torch.maximum(now, was)
                h = slice(at, at + old - start)
                step = half_step(V[pg, h] / now[:, None], code) * now[:, None]
                E[pg, h] = torch.where((now > was)[:, None], step, 0.0)
            S[pg, at // block] = now
            h = slice(at + lo - start, at + hi - start)
            V[pg, h] = part
            E[pg, h] = half_step(part / now[:, None], code) * now[:, None] * (1 + 2 ** -20) + err[r]
        t0 += n
    return V, E, S


def weights(b, before, causal=True, scale=None):
    """(sums, bound) in float64: `before` plus every seen token's softmax weights.  Bound: a
    weight is off by its score's error (products exact, hd float32 sums, 2^-23 of them each)
    twice (itself and the sum), 2^-17 for exponential, sum and division; one rounding a row
    of the running sums; float32 exponentials below 2^-126, the least normal number, are 0, so
    that each of the rows may miss up to that."""
    q, page = b["q"].double(), b["page"]
    T, Hq, hd = q.shape
    Hkv = b["k"].shape[2]
    G = Hq // Hkv
    scale = hd ** -0.5 if scale is None else scale
    out, bound = before.double().clone(), torch.zeros_like(before, dtype=torch.float64)
    t0 = 0
    for s, (n, m) in enumerate(zip(b["new"], b["m"])):
        if n and m:
            idx = torch.arange(m, device=q.device)
            pg, st = b["table"][s][idx // page].long(), idx % page
            ok = (pg >= 0) & (pg < b["k"].shape[0])
            K = torch.where(ok[:, None, None], b["k"][pg.clamp(0, b["k"].shape[0] - 1), st].double(), 0.0)
            i = torch.arange(n, device=q.device)[:, None]
            see = idx[None] <= m - n + i if causal else torch.ones(n, m, dtype=torch.bool,
                                                                   device=q.device)
            for c in range(Hkv):
                add = torch.zeros(m, dtype=torch.float64, device=q.device)
                err = torch.zeros_like(add)
                for h in range(c * G, (c + 1) * G):
                    Q = q[t0:t0 + n, h]
                    S = (Q @ K[:, c].T * scale).masked_fill(~see, -math.inf)
                    P = torch.softmax(S, -1).masked_fill(~see, 0.0)
                    d = (2.0 ** -23 * hd * scale * (Q.abs() @ K[:, c].abs().T)).masked_fill(~see, 0.0)
                    d = d.amax(-1, keepdim=True)
                    add += P.sum(0)
                    err += (P * (2 * d + 2.0 ** -17)).sum(0)
                w = torch.zeros_like(out[0, 0, 0]) + add
                out[pg[ok], c, st[ok]] += w[ok]
                bound[pg[ok], c, st[ok]] = (err + n * G * 2.0 ** -126 + 2.0 ** -23 * (n * G + 1) * out[pg.clamp(0, out.shape[0] - 1), c, st].abs())[ok]
        t0 += n
    return out, bound


def evict(b, w, keep, first, last):
    """What cache_evict leaves, in plain Python: a dict of tensors."""
    page = b["page"]
    eight = "k_scale" in b
    B, Hkv = len(b["m"]), b["k"].shape[2]
    raw = {x: b[x].clone().view(torch.uint8 if eight else torch.int16) for x in "kv"}
    src = {x: t.clone() for x, t in raw.items()}
    out = {"w": w.clone(), "kept": torch.full((B, Hkv, keep), -1, dtype=torch.int32),
           "lens": b["kv_lens"].clone()}
    if eight:
        out.update(k_scale=b["k_scale"].clone(), v_scale=b["v_scale"].clone())
    cols = b["table"].shape[1]
    pages = b["k"].shape[0]
    for s, m in enumerate(b["m"]):
        m = min(m, cols * page)
        if m <= keep:
            for h in range(Hkv):
                out["kept"][s, h, :m] = torch.arange(m)
            continue
        out["lens"][s] = keep
        pg = [int(b["table"][s, i // page]) for i in range(m)]
        ok = [0 <= p < pages for p in pg]
        for h in range(Hkv):
            ws = [float(w[pg[i], h, i % page]) if ok[i] else 0.0 for i in range(m)]
            key = [(-math.inf if math.isnan(x) else x, not math.isnan(x)) for x in ws]
            inner = sorted(range(first, m - last), key=lambda i: (key[i], -i), reverse=True)
            stay = list(range(first)) + sorted(inner[:keep - first - last]) + list(range(m - last, m))
            out["kept"][s, h] = torch.tensor(stay, dtype=torch.int32)
            for i in range(keep, m):
                if ok[i]:
                    out["w"][pg[i], h, i % page] = 0.0
            for to, i in enumerate(stay):
                if ok[to]:
                    out["w"][pg[to], h, to % page] = ws[i]
            for x in "kv":
                if not eight:
                    for to, i in enumerate(stay):
                        if ok[to]:
                            raw[x][pg[to], to % page, h] = src[x][pg[i], i % page, h] if ok[i] else 0
                    continue
                blk, code = b["block"], b[x].dtype
                sc = b[x + "_scale"]
                f = [float(sc[pg[i], i % page // blk, h]) if ok[i] else 0.0 for i in stay]
                for d0 in range(0, keep, blk):
                    d1 = min(keep, d0 + blk)
                    now = max(f[d0:d1])
                    if not ok[d0]:
                        continue
                    out[x + "_scale"][pg[d0], d0 % page // blk, h] = now
                    for to in range(d0, d1):
                        i = stay[to]
                        if not ok[i]:
                            row = torch.zeros(b[x].shape[3], dtype=torch.uint8)
                        else:
                            c = src[x][pg[i], i % page, h].view(code).float()
                            by = f[to] / now if now > 0 else 0.0
                            row = src[x][pg[i], i % page, h] if f[to] == now else \
                                to_codes(c * by, code).view(torch.uint8)
                        raw[x][pg[to], to % page, h] = row
    out.update(k=raw["k"], v=raw["v"])
    return out


check = R.check
