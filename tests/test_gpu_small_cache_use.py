"""The calls that make the cache smaller as a program uses them: one after the other, captured
into a graph, on other streams, over views, and where masked places hold what is no number."""
import math

import pytest
import torch

from tests import attention_ref as R
from tests import small_cache_ref as S
from tests.test_gpu_small_cache import CODES, DTYPES, batch, cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def pages(B, tokens, page, H, hd, block, code, seed=0):
    """An empty cache of codes with room for `tokens` of each of B sequences."""
    per = -(-tokens // page)
    g = torch.Generator("cpu").manual_seed(seed)
    table = torch.randperm(B * per, generator=g).int().view(B, per).cuda()
    kv = [torch.zeros(B * per, page, H, hd, device="cuda").to(code) for _ in "kv"]
    sc = [torch.full((B * per, page // block, H), math.nan, device="cuda") for _ in "kv"]
    return {"k": kv[0], "v": kv[1], "k_scale": sc[0], "v_scale": sc[1], "table": table,
            "kv_lens": torch.zeros(B, dtype=torch.int32, device="cuda"), "block": block,
            "page": page}


@pytest.mark.parametrize("code", CODES)
def test_prompt_weights_eviction_and_decoding(sls, code):
    """A ragged batch of prompts is appended and attended, its last tokens vote, the cache is cut,
    and new tokens are decoded, weighed and cut again: every step against float64 over the codes
    that the steps before left."""
    B, Hq, Hkv, hd, page, block, dt = 3, 8, 2, 64, 32, 16, torch.bfloat16
    new = [150, 70, 33]
    b = pages(B, 160, page, Hkv, hd, block, code)
    w = torch.zeros(b["k"].shape[0], Hkv, page, device="cuda")
    g = torch.Generator("cuda").manual_seed(5)
    rope = sls.Rope.make(hd, base=1e5)
    T = sum(new)
    x = torch.randn(T, Hq + 2 * Hkv, hd, generator=g, device="cuda").to(dt)
    cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    b["kv_lens"] += torch.tensor(new, dtype=torch.int32, device="cuda")
    q = sls.qkv_append_q8(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *cache(b), cu_seqlens=cu,
                          rope=rope)
    ref = dict(b, q=q, new=new, m=new)
    want, bound = R.attention(S.plain(ref))
    S.check(sls.attention_prefill_q8(q, *cache(b), cu), want, bound, "prompt")
    # the last eight tokens of each prompt vote
    vote = torch.cat([q[cu[s + 1] - 8:cu[s + 1]] for s in range(B)])
    cu8 = torch.arange(0, 8 * B + 1, 8, dtype=torch.int32, device="cuda")
    ref = dict(b, q=vote, new=[8] * B, m=new)
    want, bound = S.weights(S.plain(ref), w)
    sls.attention_weights(vote, b["k"], b["table"], b["kv_lens"], w, cu_seqlens=cu8,
                          k_scale=b["k_scale"])
    S.check(w, want, bound, "votes")
    at = torch.tensor(new, device="cuda")
    for keep in (40, 24):
        before = {k: (v.cpu() if torch.is_tensor(v) else v) for k, v in b.items()}
        before["m"] = b["kv_lens"].tolist()
        want = S.evict(before, w.cpu(), keep, 4, 8)
        kept = sls.cache_evict(b["k"], b["v"], b["table"], b["kv_lens"], w, keep, first=4, last=8,
                               k_scale=b["k_scale"], v_scale=b["v_scale"])
        assert torch.equal(kept.cpu(), want["kept"])
        assert b["kv_lens"].tolist() == [min(keep, m) for m in before["m"]]
        assert torch.equal(b["k"].cpu().view(torch.uint8), want["k"])
        # decode three tokens at the positions that follow the uncut prompt
        for i in range(3):
            y = torch.randn(B, Hq + 2 * Hkv, hd, generator=g, device="cuda").to(dt)
            b["kv_lens"] += 1
            q = sls.qkv_append_q8(y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:], *cache(b),
                                  positions=at.int(), rope=rope)
            at += 1
            m = b["kv_lens"].tolist()
            ref = S.plain(dict(b, q=q, new=[1] * B, m=m))
            want, bound = R.attention(ref)
            S.check(sls.attention_decode_q8(q, *cache(b)), want, bound, "decode")
            want, bound = S.weights(ref, w)
            sls.attention_weights(q, b["k"], b["table"], b["kv_lens"], w, k_scale=b["k_scale"])
            S.check(w, want, bound, "weights")


def steps(sls, b, q, k, v, w, ws, keep):
    """One decoding step and a cut; everything that it writes."""
    out = sls.qkv_append_q8(q, k, v, *cache(b))
    o = sls.attention_decode_q8(out, *cache(b), workspace=ws)
    sls.attention_weights(out, b["k"], b["table"], b["kv_lens"], w, k_scale=b["k_scale"], workspace=ws)
    cu = b["one"]
    p = sls.attention_prefill_q8(out, *cache(b), cu, workspace=ws)
    kept = sls.cache_evict(b["k"], b["v"], b["table"], b["kv_lens"], w, keep, first=1, last=2,
                           k_scale=b["k_scale"], v_scale=b["v_scale"])
    return [out, o, p, kept, w, b["k"], b["v"], b["k_scale"], b["v_scale"], b["kv_lens"]]


def copy_of(b):
    return {k: (v.clone() if torch.is_tensor(v) else v) for k, v in b.items()}


def same(a, c):
    return all(torch.equal(x.view(torch.uint8) if x.element_size() == 1 else
                           x.nan_to_num(nan=7.0) if x.is_floating_point() else x,
                           y.view(torch.uint8) if y.element_size() == 1 else
                           y.nan_to_num(nan=7.0) if y.is_floating_point() else y)
               for x, y in zip(a, c))


@pytest.mark.parametrize("code", CODES)
def test_captured_and_replayed(sls, code):
    """Two graphs that share a workspace, replayed in turn on new contents, and the same on a
    stream of its own: the bits of calls one by one."""
    m, Hq, Hkv, hd = [70, 3, 200], 16, 4, 128
    b = batch([1] * 3, m, Hq, Hkv, hd, 32, 16, torch.bfloat16, code, seed=21)
    b["one"] = torch.arange(4, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    w0 = torch.rand(b["k"].shape[0], Hkv, 32, generator=g, device="cuda")
    qkv = [torch.randn(3, Hq + 2 * Hkv, hd, generator=g, device="cuda").bfloat16() for _ in range(3)]
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")

    def parts(x):
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    want = []
    for x in qkv:
        want.append([t.clone() for t in steps(sls, copy_of(b), *parts(x), w0.clone(), ws, 50)])
    graphs = []
    for _ in range(2):
        own, w, x = copy_of(b), w0.clone(), qkv[0].clone()
        steps(sls, copy_of(b), *parts(x), w0.clone(), ws, 50)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = steps(sls, own, *parts(x), w, ws, 50)
        graphs.append((graph, own, w, x, got))
    for turn in range(3):
        for graph, own, w, x, got in graphs:
            for key, t in own.items():
                if torch.is_tensor(t):
                    t.copy_(b[key])
            w.copy_(w0)
            x.copy_(qkv[turn])
            graph.replay()
            torch.cuda.synchronize()
            assert same(got, want[turn])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = steps(sls, copy_of(b), *parts(qkv[1]), w0.clone(), ws, 50)
    side.synchronize()
    assert same(got, want[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_views(sls, dtype):
    """Heads outside slots, scales and weights that are parts of larger tensors, queries that are
    slices, pages of one head among others."""
    new, m, Hq, Hkv, hd, page = [3, 40], [60, 300], 6, 3, 96, 32
    b = batch(new, m, Hq, Hkv, hd, page, 16, dtype, torch.int8, seed=4)
    want, bound = R.attention(S.plain(b))
    n = b["k"].shape[0]

    def heads_first(t):  # pages x heads x slots x elements, seen as pages x slots x heads x elements
        return t.transpose(1, 2).contiguous().transpose(1, 2)

    def among(t):
        big = torch.full((n, t.shape[1] + 1, Hkv + 2), math.nan, device="cuda")
        big[:, 1:, 1:Hkv + 1] = t
        return big[:, 1:, 1:Hkv + 1]

    v = dict(b, k=heads_first(b["k"]), v=heads_first(b["v"]), k_scale=among(b["k_scale"]),
             v_scale=among(b["v_scale"]))
    q = torch.zeros(sum(new), Hq + 5, hd, dtype=dtype, device="cuda")
    q[:, 2:Hq + 2] = b["q"]
    q = q[:, 2:Hq + 2]
    S.check(sls.attention_prefill_q8(q, *cache(v), b["cu"]), want, bound, "prefill")
    one = dict(b, q=b["q"][:2].contiguous(), new=[1, 1])
    want, bound = R.attention(S.plain(one), causal=False)
    S.check(sls.attention_decode_q8(q[:2], *cache(v)), want, bound, "decode")
    big = torch.zeros(n, Hkv + 1, page + 4, device="cuda")
    w = big[:, :Hkv, :page]
    want, bound = S.weights(S.plain(b), torch.zeros_like(w))
    sls.attention_weights(q, v["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                          k_scale=v["k_scale"])
    S.check(w, want, bound, "weights")
    assert not big[:, Hkv].any() and not big[:, :, page:].any()
    # the same cut of both layouts
    x = torch.rand(n, Hkv, page, device="cuda")
    w.copy_(x)
    twin = copy_of(b)
    kept = sls.cache_evict(twin["k"], twin["v"], b["table"], twin["kv_lens"], x, 33, first=2, last=5,
                           k_scale=twin["k_scale"], v_scale=twin["v_scale"])
    lens = b["kv_lens"].clone()
    again = sls.cache_evict(v["k"], v["v"], b["table"], lens, w, 33, first=2, last=5,
                            k_scale=v["k_scale"], v_scale=v["v_scale"])
    assert torch.equal(kept, again) and torch.equal(lens, twin["kv_lens"]) and torch.equal(w, x)
    assert same([v["k"], v["v"], v["k_scale"], v["v_scale"]],
                [twin["k"], twin["v"], twin["k_scale"], twin["v_scale"]])


def test_hidden_tokens_that_are_no_numbers(sls):
    """NaN codes, NaN and infinite scales where a row does not look leave its result alone."""
    new, m = [40, 20], [100, 20]
    b = batch(new, m, 8, 2, 64, 32, 16, torch.bfloat16, torch.float8_e4m3fn, seed=9)
    clean = sls.attention_prefill_q8(b["q"], *cache(b), b["cu"])
    w = torch.zeros(b["k"].shape[0], 2, 32, device="cuda")
    sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                          k_scale=b["k_scale"])
    assert w.isfinite().all() and clean.isfinite().all()
    for s, last in enumerate(m):
        pg, slot = int(b["table"][s, (last - 1) // 32]), (last - 1) % 32
        for x in "kv":
            b[x].view(torch.uint8)[pg, slot] = 0x7f
    out = sls.attention_prefill_q8(b["q"], *cache(b), b["cu"])
    seen = torch.zeros(sum(new), dtype=torch.bool)
    seen[torch.tensor(new).cumsum(0) - 1] = True
    assert torch.equal(out[~seen.cuda()], clean[~seen.cuda()])
    assert out[seen.cuda()].isnan().all()
    # only the last rows see those tokens: without them (their queries' rows left out) the sums
    # are numbers
    front = torch.cat([b["q"][:39], b["q"][40:59]])
    cu = torch.tensor([0, 39, 58], dtype=torch.int32, device="cuda")
    lens = b["kv_lens"] - 1
    v = torch.zeros_like(w)
    sls.attention_weights(front, b["k"], b["table"], lens, v, cu_seqlens=cu, k_scale=b["k_scale"])
    assert v.isfinite().all() and (v.sum() - 58 * 8).abs() < 1e-3 * 58 * 8


def test_weights_of_rows_that_are_no_numbers(sls):
    """A NaN query leaves NaN on the tokens that it sees, of its own sequence and key head only."""
    for new in ([1, 1], [40, 40]):
        m = [64, 64]
        b = R.make_batch(new, m, 8, 2, 64, 16, torch.float16, seed=2)
        b["q"][0, 5] = math.nan          # sequence 0, key head 1
        w = torch.zeros(b["k"].shape[0], 2, 16, device="cuda")
        sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"])
        first = b["table"][0, :4].long()
        see = 64 - new[0] + 1
        got = w[first, 1].reshape(-1)
        assert got[:see].isnan().all() and got[see:].isfinite().all()
        assert w[first, 0].isfinite().all()
        assert w[b["table"][1, :4].long()].isfinite().all()


def test_nothing_to_do(sls):
    b = batch([1], [20], 4, 2, 64, 16, 16, torch.bfloat16, torch.int8, seed=1)
    none = dict(b, table=b["table"][:0], kv_lens=b["kv_lens"][:0])
    q, cu = b["q"][:0], torch.zeros(1, dtype=torch.int32, device="cuda")
    w = torch.ones(b["k"].shape[0], 2, 16, device="cuda")
    assert sls.attention_decode_q8(q, *cache(none)).shape == q.shape
    assert sls.attention_prefill_q8(q, *cache(none), cu).shape == q.shape
    x = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    assert sls.qkv_append_q8(x[:, :4], x[:, 4:6], x[:, 6:], *cache(none)).shape == q.shape
    sls.attention_weights(q, b["k"], none["table"], none["kv_lens"], w, k_scale=b["k_scale"])
    sls.attention_weights(q, b["k"], b["table"], b["kv_lens"], w, cu_seqlens=torch.zeros_like(cu).repeat(2),
                          k_scale=b["k_scale"])
    kept = sls.cache_evict(b["k"], b["v"], none["table"], none["kv_lens"], w, 4, k_scale=b["k_scale"],
                           v_scale=b["v_scale"])
    assert kept.shape == (0, 2, 4) and (w == 1).all()
    # empty sequences
    b["kv_lens"].zero_()
    assert not sls.attention_decode_q8(b["q"], *cache(b)).any()
    sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, k_scale=b["k_scale"])
    assert (w == 1).all()


@pytest.mark.parametrize("length", [5000, 131072, 400000])
def test_evict_long(sls, length):
    """Few heads of long sequences: clusters, and past what they hold the way of any length."""
    page, Hkv, hd, keep = 128, 1, 16, 3001
    n = -(-length // page)
    g = torch.Generator("cuda").manual_seed(length)
    table = torch.randperm(n, generator=g, device="cuda").int().view(1, n)
    k = torch.randint(-99, 99, (n, page, Hkv, hd), generator=g, device="cuda").half()
    v = torch.randint(-99, 99, (n, page, Hkv, hd), generator=g, device="cuda").half()
    w = (torch.rand(n, Hkv, page, generator=g, device="cuda") * 5000).round()  # many equal ones
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    at = table[0].long()

    def flat(t):
        return t[at].reshape(n * page, -1)[:length]

    kf, vf, wf = flat(k).clone(), flat(v).clone(), w[at, 0].reshape(-1)[:length].clone()
    rank = wf.clone()
    rank[:7] = rank[length - 11:] = math.inf
    idx = torch.sort(rank, descending=True, stable=True).indices[:keep].sort().values
    kept = sls.cache_evict(k, v, table, lens, w, keep, first=7, last=11)
    assert torch.equal(kept[0, 0].long(), idx) and lens.item() == keep
    assert torch.equal(flat(k)[:keep], kf[idx]) and torch.equal(flat(v)[:keep], vf[idx])
    assert torch.equal(flat(k)[keep:], kf[keep:])
    now = w[at, 0].reshape(-1)[:length]
    assert torch.equal(now[:keep], wf[idx]) and not now[keep:].any()


def test_many_sequences(sls):
    """More sequences than a CTA has threads, most of them short: packed calls and single tokens."""
    B = 700
    g = torch.Generator("cpu").manual_seed(3)
    m = torch.randint(0, 40, (B,), generator=g).tolist()
    b = batch([1] * B, m, 2, 1, 32, 16, 16, torch.float16, torch.int8, seed=5)
    want, bound = R.attention(S.plain(b), causal=False)
    S.check(sls.attention_decode_q8(b["q"], *cache(b)), want, bound, "decode")
    w = torch.zeros(b["k"].shape[0], 1, 16, device="cuda")
    want, bound = S.weights(S.plain(b), w)
    sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                          k_scale=b["k_scale"])
    S.check(w, want, bound, "weights")
    w = torch.rand(b["k"].shape[0], 1, 16, device="cuda")
    host = {k: (v.cpu() if torch.is_tensor(v) else v) for k, v in b.items()}
    ref = S.evict(host, w.cpu(), 20, 1, 1)
    kept = sls.cache_evict(b["k"], b["v"], b["table"], b["kv_lens"], w, 20, first=1, last=1,
                           k_scale=b["k_scale"], v_scale=b["v_scale"])
    assert torch.equal(kept.cpu(), ref["kept"]) and torch.equal(w.cpu(), ref["w"])
    assert torch.equal(b["k"].cpu().view(torch.uint8), ref["k"])


@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_of_many_rows(sls, dtype):
    """More rows than two tiles, of a group that does not divide 128, over several tiles of tokens;
    large scores."""
    for scale in (None, 2.0):
        b = R.make_batch([200, 77], [500, 300], 21, 3, 128, 64, dtype, seed=8)
        w = torch.zeros(b["k"].shape[0], 3, 64, device="cuda")
        want, bound = S.weights(b, w, scale=scale)
        sls.attention_weights(b["q"], b["k"], b["table"], b["kv_lens"], w, cu_seqlens=b["cu"],
                              scale=scale)
        S.check(w, want, bound, f"scale {scale}")


def test_eviction_that_keeps_as_many_as_there_can_be(sls):
    """kept has 2^31 - 1 places for a sequence of 40 tokens: every other one is -1, and nothing
    outside is written."""
    k = torch.zeros(3, 16, 1, 16, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
    lens = torch.tensor([40], dtype=torch.int32, device="cuda")
    w = torch.rand(3, 1, 16, device="cuda")
    before = w.clone()
    kept = sls.cache_evict(k, k.clone(), table, lens, w, 2 ** 31 - 1)
    assert kept.shape == (1, 1, 2 ** 31 - 1)
    assert kept[0, 0, :40].tolist() == list(range(40))
    assert kept[0, 0, 40:].min().item() == -1 and kept[0, 0, 40:].max().item() == -1
    assert lens.tolist() == [40] and torch.equal(w, before)
