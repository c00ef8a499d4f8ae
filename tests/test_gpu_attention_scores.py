"""Scores far from zero: what weighs is their distance from the row's largest."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attention_not_finite import equal_scores

pytestmark = pytest.mark.gpu


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


# one cluster; many clusters' worth of keys, cut into parts; more query heads than a tile has rows
ONE = [(([1], [700], 8, 2, 128, 64)), (([1], [40000], 4, 2, 64, 64)), (([1], [900], 17, 1, 128, 32))]


@pytest.mark.parametrize("score", [torch.finfo(torch.bfloat16).min / 8, -3.0e9, 1.0e6, 2.0e30])
@pytest.mark.parametrize("case", ONE)
def test_decode_scores_far_from_zero(sls, case, score):
    b = R.make_batch(*case, torch.bfloat16, seed=15)
    want, bound = equal_scores(b, score)
    R.check(decode(sls, b, scale=1.0), want, bound)


@pytest.mark.parametrize("start", [0.0, 640.0, -2.0 ** 20, 2.0 ** 20])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("call,case", [("decode", c) for c in ONE] +
                         [("prefill", ([130], [260], 4, 2, 64, 64)),
                          ("prefill", ([40], [5000], 4, 2, 64, 16))])
def test_scores_from_any_start(sls, call, case, dtype, start):
    """Scores start + 0 .. 7, exact in float32 and in their 16-bit factors.  The bound: the
    weights' and the result's rounding to 16 bits, 2^-15 for exponentials and sums, and 2^-13
    for the rounding of the scaled maximum, 2^-24 of at most 1024 twice (beyond that the
    distance is formed first)."""
    b = R.make_batch(*case, dtype, seed=19)
    b["q"].zero_()
    b["q"][..., 0] = 1024.0
    b["q"][..., 1] = 1.0
    g = torch.Generator("cuda").manual_seed(21)
    b["k"][..., 0] = start / 1024.0
    b["k"][..., 1] = torch.randint(0, 8, b["k"].shape[:3], generator=g, device="cuda").to(dtype)
    want, _ = R.attention(b, True, 1.0)
    size, _ = R.attention(dict(b, v=b["v"].abs()), True, 1.0)
    u = R.U[dtype]
    bound = u * want.abs() + (u + 2.0 ** -13 + 2.0 ** -15) * size + 2 * R.TINY[dtype]
    R.check((decode if call == "decode" else prefill)(sls, b, scale=1.0), want, bound)


@pytest.mark.parametrize("low", [-24.5, -26.0, -28.5])
@pytest.mark.parametrize("call", ["decode", "prefill"])
def test_many_small_weights(sls, call, low):
    """One key of weight 1 whose value is 0 and 131072 of weight 2^low, float16: all that the
    output holds comes from the small weights, which only the sum would count if they
    rounded to 0.  As many sequences (of the same pages) as keep each in one piece, where the
    large key's maximum holds for all.

    The bound, relative to an output whose terms have one sign: 2 u for the roundings of
    weights and result, 2^-15 for exponentials, 2^-23 for each of the tensor cores'
    additions of 16 keys (which may truncate), 2^-24 for each of the sum's additions of at
    least 32 keys; and half the smallest float16 step, 2^-25, for each weight times its value,
    carried 2^15 (decode) and at least 2^7 (prefill) up."""
    m, B = 131073, 610 if call == "decode" else 160
    b = R.make_batch([1], [m], 4, 2, 64, 128, torch.float16, seed=23)
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    b["k"][..., 0] = low
    b["v"].abs_()
    first = b["table"][0, 0].long()
    b["k"][first, 0, :, 0] = 0.0
    b["v"][first, 0] = 0.0
    scale = 0.6931471805599453
    want, _ = R.attention(b, True, scale)
    V = R.gather(b["v"], b["table"][0], m, 128).double().sum(0)
    step = 2.0 ** -25 * 2.0 ** (-15 if call == "decode" else -7)
    rel = 2 * R.U[torch.float16] + 2.0 ** -15 + (m / 16 + 1) * 2.0 ** -23 + (m / 32 + 1) * 2.0 ** -24
    # results below 2^-14 are rounded to float16's smallest step
    bound = rel * want.abs() + step * V.repeat_interleave(2, 0)[None] + R.TINY[torch.float16]
    many = dict(b, q=b["q"].repeat(B, 1, 1), table=b["table"].repeat(B, 1),
                kv_lens=b["kv_lens"].repeat(B),
                cu=torch.arange(B + 1, dtype=torch.int32, device="cuda"))
    got = (decode if call == "decode" else prefill)(sls, many, scale=scale)
    R.check(got, want.expand(B, -1, -1), bound.expand(B, -1, -1))
