"""The attention calls at the sizes at which their kernels go on from one piece of work to
the next: prefill with several items a CTA, append with several tokens a CTA, many sequences,
and appends of one token per sequence without offsets.  Against the float64 statement; slots
that no sequence covers hold NaN."""
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


# ---------------------------------------------------------------------------
# prefill: more items than SMs
# ---------------------------------------------------------------------------

RAGGED = [700, 1, 0, 333, 1500, 64, 129, 2000, 5]
BEHIND = [0, 50, 20, 0, 3, 700, 0, 100, 0]

PREFILL = [
    # new, m, Hq, Hkv, hd, page, causal, items (pairs of query tiles times key heads)
    ([2048], [2048], 28, 4, 128, 64, True, 228),
    ([3701], [3800], 12, 12, 64, 32, True, 180),
    ([2500], [2500], 16, 16, 64, 128, True, 160),
    (RAGGED, [n + h for n, h in zip(RAGGED, BEHIND)], 16, 16, 64, 16, True, 368),
    (RAGGED, [n + h for n, h in zip(RAGGED, BEHIND)], 24, 8, 128, 64, True, 480),
    (RAGGED, [n + h for n, h in zip(RAGGED, BEHIND)], 16, 8, 128, 16, False, 320),
    # rows before the first key and sequences without keys among longer ones
    ([600, 300, 900, 40], [600, 120, 0, 1000], 16, 16, 80, 32, True, 160),
    # more sequences than a warp has lanes
    ([1 + 5 * i for i in range(60)], [1 + 5 * i + (i % 7) * 40 for i in range(60)], 8, 8, 64, 16,
     True, 544),
    ([20] * 1024, [20 + i % 30 for i in range(1024)], 4, 2, 64, 16, True, 2048),
]


def items(new, Hq, Hkv):
    pair = 2 * (128 // (Hq // Hkv))
    return Hkv * sum(-(-n // pair) for n in new)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", PREFILL, ids=lambda c: f"{len(c[0])}x{c[2]}-{c[3]}x{c[4]}")
def test_prefill_of_many_items(sls, case, dtype):
    new, m, Hq, Hkv, hd, page, causal, least = case
    assert items(new, Hq, Hkv) >= least
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=len(str(case)))
    want, bound = R.attention(b, causal)
    got = sls.attention_prefill(b["q"], b["k"], b["v"], b["table"], b["kv_lens"], b["cu"],
                                causal=causal)
    R.check(got, want, bound)
    assert sls.attention_status() == 0


# ---------------------------------------------------------------------------
# append: 2, 4 and 8 tokens a CTA, partial last tiles
# ---------------------------------------------------------------------------

MODES = [
    # hd, pairs, interleaved, norm
    (128, 64, False, True),       # halves of whole vectors
    (128, 48, True, True),        # pairs side by side
    (80, 12, False, True),        # halves that split vectors
    (64, 32, False, False),
    (64, 9, False, True),
    (64, 0, False, True),         # no rotation
]


def appended(sls, b, x, Hq, Hkv, positions, mode, dtype, cu):
    hd, pairs, interleaved, norm = mode
    g = torch.Generator("cuda").manual_seed(31)
    qw = kw = None
    if norm:
        qw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
        kw = (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).to(dtype)
    f = sls.Rope.make(max(2, 2 * pairs), base=1e6).inv_freq[:pairs].contiguous()
    rope = sls.Rope(f, interleaved=interleaved, scale=0.75) if pairs else None
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    qo, K, V, qb, bK = R.append(q, k, v, b, positions, qw, kw, 1e-5, f if pairs else None,
                                interleaved, 0.75)
    got = sls.qkv_append(q, k, v, b["k"], b["v"], b["table"], b["kv_lens"], cu_seqlens=cu,
                         positions=positions, q_weight=qw, k_weight=kw, eps=1e-5, rope=rope)
    R.check(got, qo, qb, "q")
    hole = torch.isnan(K)
    assert torch.equal(torch.isnan(b["k"]), hole) and torch.equal(torch.isnan(b["v"]), hole)
    R.check(b["k"].double().masked_fill(hole, 0), K.masked_fill(hole, 0), bK.masked_fill(hole, 0),
            "k")
    assert torch.equal(b["v"].double().masked_fill(hole, 0), V.masked_fill(hole, 0))


def projected(T, Hq, Hkv, hd, dtype):
    g = torch.Generator("cuda").manual_seed(37)
    x = torch.randn(T, Hq + 2 * Hkv, hd, generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, 131072, (T,), generator=g, device="cuda", dtype=torch.int32)
    return x, pos


@pytest.mark.parametrize("T", [1303, 2501, 5003])
@pytest.mark.parametrize("mode", MODES)
def test_append_of_several_tokens_a_cta(sls, T, mode):
    dtype = DTYPES[T % 2 if mode[3] else 1 - T % 2]
    new = [T - 700, 0, 1, 402, 297]
    m = [T - 700 + 33, 9, 1, 200, 1000]              # the fourth has more tokens than places
    b = R.make_batch(new, m, 6, 2, mode[0], 32, dtype, seed=41)
    x, pos = projected(T, 6, 2, mode[0], dtype)
    appended(sls, b, x, 6, 2, pos, mode, dtype, b["cu"])


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("B,mode", [(3, MODES[0]), (5, MODES[1]), (2, MODES[2]), (700, (64, 8, False, True)),
                                    (1303, (64, 8, False, True))])
def test_append_of_one_token_per_sequence(sls, B, mode, given):
    """Without offsets token s goes to the last place of sequence s."""
    m = [1 + (37 * s) % 301 for s in range(B)]
    b = R.make_batch([1] * B, m, 4, 2, mode[0], 64, torch.bfloat16, seed=43)
    x, pos = projected(B, 4, 2, mode[0], torch.bfloat16)
    appended(sls, b, x, 4, 2, pos if given else None, mode, torch.bfloat16, None)


@pytest.mark.parametrize("causal", [True, False])
def test_lengths_up_to_the_largest_integer(sls, causal):
    """A length is cut to what the page table holds, whatever it says: rows of new tokens
    past the table see all of it, and the batch's other sequences theirs."""
    table_tokens = 512
    for n in (30, 300):
        b = R.make_batch([n, 200, 33], [table_tokens, 200, 77], 4, 2, 64, 16, torch.bfloat16, seed=47)
        b["table"] = b["table"][:, :table_tokens // 16].contiguous()
        b["kv_lens"][0] = (1 << 31) - 1
        all_of_it = dict(b, q=b["q"][:n], new=[n], m=[table_tokens])
        want, bound = R.attention(all_of_it, False)
        rest = dict(b, q=b["q"][n:], new=[200, 33], m=[200, 77], table=b["table"][1:])
        want2, bound2 = R.attention(rest, causal)
        out = torch.full_like(b["q"], float("nan"))
        sls.attention_prefill(b["q"], b["k"], b["v"], b["table"], b["kv_lens"], b["cu"],
                              causal=causal, out=out)
        R.check(out, torch.cat([want, want2]), torch.cat([bound, bound2]))
        assert sls.attention_status() == 0
