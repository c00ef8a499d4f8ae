"""Rotation at any position: the angle is that of the exact product of position and
frequency, past the integers that float32 holds too."""
import math
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu

TWO_PI = Decimal("6.283185307179586476925286766559005768394338798750211641949889184615632812572")


@pytest.fixture(scope="module")
def sls():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_19368_gb300 as sls
    return sls


def angle(p, f):
    """p f modulo 2 pi, f the float32 itself."""
    getcontext().prec = 70
    x = Fraction(p) * Fraction(f)
    d = Decimal(x.numerator) / Decimal(x.denominator)
    return float(d - TWO_PI * (d / TWO_PI).to_integral_value())


POSITIONS = [0, 1, -1, 131071, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, (1 << 24) + 3, 33554435,
             -(1 << 24) - 1, 123456789, -123456789, 1 << 30, (1 << 30) + 7, (1 << 31) - 65,
             (1 << 31) - 1, -(1 << 31), -(1 << 31) + 1]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("given", [True, False])
def test_angles_at_any_position(sls, given, interleaved):
    """`given`: positions as an argument, or the cache index of tokens of a long sequence (its
    pages beyond the new tokens' are not read)."""
    hd, half = 64, 32
    T = len(POSITIONS)
    f = torch.tensor([1.0, 0.999, 3.0, 100.5] + [1e6 ** (-i / 28) for i in range(28)],
                     dtype=torch.float32)
    g = torch.Generator().manual_seed(51)
    x = torch.randn(T, 4, hd, generator=g).half()
    rope = sls.Rope(f.cuda(), interleaved=interleaved)
    if given:
        pos = POSITIONS
        b = R.make_batch([T], [T], 2, 1, hd, 64, torch.float16, seed=53)
        table, lens = b["table"], b["kv_lens"]
        positions = torch.tensor(pos, dtype=torch.int64).to(torch.int32).cuda()
    else:
        m = (1 << 24) + 5
        pos = list(range(m - T, m))
        b = R.make_batch([T], [T], 2, 1, hd, 64, torch.float16, seed=53)
        table = b["table"][:, :1].expand(1, m // 64 + 1).contiguous()
        lens = torch.tensor([m], dtype=torch.int32, device="cuda")
        positions = None
    xc = x.cuda()
    got = sls.qkv_append(xc[:, :2], xc[:, 2:3], xc[:, 3:], b["k"], b["v"], table, lens,
                         cu_seqlens=b["cu"], positions=positions, rope=rope)
    t = torch.tensor([[angle(p, v) for v in f.tolist()] for p in pos], dtype=torch.float64)
    a = x[:, :2].double()
    even = a[..., 0::2] if interleaved else a[..., :half]
    odd = a[..., 1::2] if interleaved else a[..., half:]
    c, s = t.cos()[:, None], t.sin()[:, None]
    turned = [even * c - odd * s, odd * c + even * s]
    size = even.abs() + odd.abs()
    join = (lambda u, v: torch.stack([u, v], -1).flatten(-2)) if interleaved else (
        lambda u, v: torch.cat([u, v], -1))
    want = join(*turned)
    # one rounding to 16 bits, 2^-19 of the rotation's terms for cosine, sine and products
    bound = R.U[torch.float16] * want.abs() + 2.0 ** -19 * join(size, size) + R.TINY[torch.float16]
    R.check(got.cpu(), want, bound)
    assert math.isclose(angle(1, 1.0), 1.0)
