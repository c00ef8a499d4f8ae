"""Prefill over caches whose values are not all finite: every element keeps the value
that the keys its row sees give it, whatever the hidden ones hold, at the price of a
finite call."""
import math

import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def prefill(sls, b, **kw):
    return sls.attention_prefill(b["q"], b["k"], b["v"], b["table"], b["kv_lens"], b["cu"], **kw)


def put(b, what, s, x, head, element, value):
    """Element of the key or value at cache index x of sequence s."""
    page = b["table"][s, x // b["page"]].long()
    b[what][page, x % b["page"], head, element] = value


CASES = [
    # new, m, Hq, Hkv, hd, page, causal: groups of 1 (256 tokens a pair of tiles) to 66 (2)
    ([300], [300], 4, 4, 128, 64, True),
    ([700], [833], 2, 2, 64, 16, True),
    ([150, 40], [290, 40], 5, 1, 128, 16, True),
    ([200], [330], 28, 4, 128, 64, True),
    ([130], [260], 9, 3, 96, 32, True),
    ([90], [200], 66, 1, 32, 64, True),
    ([64, 10], [20, 300], 4, 2, 64, 16, True),      # rows before the first key
    ([300, 50], [300, 333], 4, 2, 64, 32, False),
    # cut into pieces and joined
    ([40], [5000], 4, 2, 64, 16, True),
    ([300], [2500], 2, 2, 128, 64, True),
    ([3, 0, 200, 1], [2500, 40, 2300, 6000], 8, 2, 128, 16, True),
    ([64], [5000], 10, 2, 64, 128, False),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", CASES)
def test_only_what_a_row_sees(sls, case, dtype):
    """Infinities and NaN at many places of the values, also next to one another and of
    both signs: an element is NaN where its row sees a NaN or both infinities, infinite
    where it sees one sign of them, and has the bits of the call with zeros in their
    places otherwise.  q is small, so that no weight falls out of the 16-bit range."""
    new, m, Hq, Hkv, hd, page, causal = case
    b = R.make_batch(new, m, Hq, Hkv, hd, page, dtype, seed=3, q_scale=0.5)
    g = torch.Generator().manual_seed(5)
    bads = []
    for s, (n, length) in enumerate(zip(new, m)):
        if n == 0 or length == 0:
            continue
        # the last key, around the first token's limit, and anywhere
        at = [length - 1, max(0, length - n), max(0, length - n // 2 - 1),
              max(0, length - n // 2 - 2), min(length - 1, 127)]
        at += torch.randint(0, length, (6,), generator=g).tolist()
        at += (max(0, length - n) + torch.randint(0, min(n, length), (12,), generator=g)).tolist()
        for x in at:
            bads.append((s, x, int(torch.randint(0, Hkv, (1,), generator=g)),
                         int(torch.randint(0, hd, (1,), generator=g)),
                         [INF, -INF, NAN][int(torch.randint(0, 3, (1,), generator=g))]))
    for s, x, h, e, _ in bads:
        put(b, "v", s, x, h, e, 0.0)
    clean = prefill(sls, b, causal=causal).double()
    want, bound = R.attention(b, causal)
    R.check(clean, want, bound)
    final = {}
    for s, x, h, e, value in bads:
        put(b, "v", s, x, h, e, value)
        final[s, x, h, e] = value
    t0 = [0]
    for n in new:
        t0.append(t0[-1] + n)
    want = clean.clone()
    G = Hq // Hkv
    for (s, x, h, e), value in final.items():
        first = max(0, x - (m[s] - new[s])) if causal else 0
        want[t0[s] + first:t0[s + 1], h * G:(h + 1) * G, e] += value
    got = prefill(sls, b, causal=causal).double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])
    assert sls.attention_status() == 0


@pytest.mark.parametrize("case", [([300], [300], 4, 2, 128, 64), ([40], [5000], 4, 2, 64, 16)])
def test_a_token_that_is_nowhere_finite(sls, case):
    """Key and value of a token all infinite or NaN: rows that do not see it keep their
    bits, rows that see it are NaN or, where its score is minus infinity, NaN in
    elements whose value is not finite (0 times infinity)."""
    new, m, Hq, Hkv, hd, page = case
    x = m[0] - 20
    for key in (INF, NAN):
        b = R.make_batch(new, m, Hq, Hkv, hd, page, torch.bfloat16, seed=7)
        clean = prefill(sls, b)
        put(b, "k", 0, x, slice(None), slice(None), 0.0)
        put(b, "k", 0, x, slice(None), 3, key)
        put(b, "v", 0, x, slice(None), slice(0, hd, 2), INF)
        got = prefill(sls, b)
        sees = x - (m[0] - new[0])
        assert torch.equal(got[:sees], clean[:sees])
        assert torch.isnan(got[sees:, :, ::2]).all()
        # with an infinite key the rows whose score is -inf do without the token
        low = (b["q"][sees:, :, 3] < 0) if key == INF else torch.zeros_like(
            b["q"][sees:, :, 3], dtype=torch.bool)
        odd = torch.isnan(got[sees:, :, 1::2])
        assert torch.equal(odd, ~low[..., None].expand_as(odd))


def test_values_of_any_size(sls):
    """Values near bfloat16's largest: the weights' sum times them stays finite although
    the maximum in use lags behind a slowly rising one."""
    b = R.make_batch([200], [256], 4, 2, 128, 64, torch.bfloat16, seed=9)
    b["v"].mul_(2.0 ** 118)
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    scale = 2.0 ** -5
    for x in range(256):                    # scores rise by 5.3 (7.7 in log2) in 128 keys
        put(b, "k", 0, x, slice(None), 0, x * 1.333)
    want, bound = R.attention(b, True, scale)
    R.check(prefill(sls, b, scale=scale), want, bound)


def equal_scores(b, score):
    """All scores of a batch `score` (before the scale of 1); what each row then is, the mean
    of the values that it sees, and a bound: the rounding of the result, and 2^-24 for each
    of the sum's additions."""
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    b["k"][..., 0] = score
    (n,), (m,) = b["new"], b["m"]
    V = R.gather(b["v"], b["table"][0], m, b["page"]).double()
    count = torch.arange(1, m + 1, device=V.device, dtype=torch.float64)[:, None, None]
    G = b["q"].shape[1] // V.shape[1]
    mean, size = ((x.cumsum(0) / count)[m - n:].repeat_interleave(G, 1) for x in (V, V.abs()))
    return mean, R.U[b["q"].dtype] * mean.abs() + (m + 8) * 2.0 ** -24 * size


@pytest.mark.parametrize("score", [torch.finfo(torch.bfloat16).min / 8, -3.0e9, 1.0e6, 2.0e30])
@pytest.mark.parametrize("case", [([130], [260], 4, 4, 64, 64), ([40], [5000], 4, 2, 64, 16)])
def test_scores_far_from_zero(sls, case, score):
    """Equal scores of any size weigh equally: what matters is their distance."""
    b = R.make_batch(*case, torch.bfloat16, seed=15)
    want, bound = equal_scores(b, score)
    R.check(prefill(sls, b, scale=1.0), want, bound)


def test_long_keys_and_other_sequences(sls):
    """An infinite value at the start of 120000 keys: seen by every row of its sequence,
    whose other elements, and the other sequences, keep their bits; no wait runs out."""
    new, m = [2000, 400], [120000, 400]
    b = R.make_batch([4, 400], [4, 400], 16, 8, 64, 64, torch.bfloat16, seed=11)
    pages = math.ceil(m[0] / 64)
    have = b["k"].shape[0]
    g = torch.Generator("cuda").manual_seed(13)
    for name in ("k", "v"):
        more = torch.randn(pages, 64, 8, 64, generator=g, device="cuda").bfloat16()
        b[name] = torch.cat([b[name], more])
    table = torch.zeros(2, pages, dtype=torch.int32, device="cuda")
    table[0] = torch.arange(have, have + pages, device="cuda")
    table[1, :b["table"].shape[1]] = b["table"][1]
    b["table"], b["m"], b["new"] = table, m, new
    b["kv_lens"] = torch.tensor(m, dtype=torch.int32, device="cuda")
    b["cu"] = torch.tensor([0, 2000, 2400], dtype=torch.int32, device="cuda")
    short = b["q"][4:]
    b["q"] = torch.cat([torch.randn(2000, 16, 64, generator=g, device="cuda").bfloat16(), short])
    clean = prefill(sls, b)
    put(b, "v", 0, 0, 3, 5, INF)
    put(b, "v", 0, 1, 3, 6, NAN)
    got = prefill(sls, b)
    assert sls.attention_status() == 0
    rows = got[:2000, 6:8]
    assert not torch.isfinite(rows[..., 5]).any() and torch.isnan(rows[..., 6]).all()
    got[:2000, 6:8, 5:7] = clean[:2000, 6:8, 5:7]
    assert torch.equal(got, clean)
    one = {"q": short, "k": b["k"], "v": b["v"], "table": table[1:].contiguous(),
           "new": [400], "m": [400], "page": 64}
    want, bound = R.attention(one)
    R.check(got[2000:], want, bound)
