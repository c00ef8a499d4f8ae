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
