"""The calls that make the cache smaller at the edges of their numbers: keys of zeros behind a norm."""
import pytest
import torch

from tests import attention_ref as R
from tests import small_cache_ref as S
from tests.test_gpu_small_cache import CODES, cache

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
