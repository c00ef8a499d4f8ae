"""Sizes past the attention calls' limits are refused, without a GPU."""
import pytest

from tests.test_attention_args import cache, rows, sls  # noqa: F401 (sls: a fixture)


@pytest.mark.parametrize("page,most", [(16, (1 << 27) - 64), (1024, (1 << 21) - 1)])
def test_page_tables_of_more_tokens_than_32_bits_count(sls, page, most):  # noqa: F811
    """Token numbers are 32 bits in the kernels: a table that could hold more, up to the
    rounding to a step or to a batch of page numbers, is refused."""
    L, r = sls.lib(), rows()
    for pages, status in ((most + 1, 2), (most + 64, 2), ((1 << 31) - 1, 2), (most, 0)):
        c = cache(sls, page_size=page, max_pages=pages, table_ld=1 << 32,
                  page_stride=page * 128, batch=0)
        assert L.sls_attention_decode(r, 4, c, 1.0, r, None, 0, None) == status
        assert L.sls_attention_prefill(r, 0, 4, c, 256, 1, 1.0, r, None, 0, None) == status
        assert L.sls_qkv_append(r, r, r, 0, 4, c, 256, None, None, None, 1e-6, None, r,
                                None) == status


def test_packed_sequences_are_limited(sls):  # noqa: F811
    """With offsets every token's or item's sequence is looked up among all of them; past the
    limit a call is refused.  One token per sequence without offsets has no such limit."""
    L, r = sls.lib(), rows()
    for batch, status in ((65536, 0), (65537, 2), (1 << 30, 2)):
        c = cache(sls, batch=batch)
        assert L.sls_attention_prefill(r, 0, 4, c, 256, 1, 1.0, r, None, 0, None) == status
        assert L.sls_qkv_append(r, r, r, 0, 4, c, 256, None, None, None, 1e-6, None, r,
                                None) == status
    # the limit is of offsets: here the count of tokens is what is wrong, not the batch
    c = cache(sls, batch=65537)
    assert L.sls_qkv_append(r, r, r, 0, 4, c, None, None, None, None, 1e-6, None, r, None) == 1
