"""What the binding of the attention calls checks and hands over, without a GPU: tensors
that say they are on one, and a library that records its calls."""
import pytest
import torch


@pytest.fixture(scope="module")
def A():
    from paper_2607_19368_gb300 import build
    build.build()
    from paper_2607_19368_gb300 import attention
    return attention


def on_gpu(t, index=0):
    """The tensor, as one of GPU `index` to those who ask."""

    class OnGpu(torch.Tensor):
        __torch_function__ = torch._C._disabled_torch_function_impl
        is_cuda = True

        def get_device(self):
            return index

    return t.as_subclass(OnGpu)


def cache_of(B=3, cols=4, index=0):
    k = on_gpu(torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16), index)
    table = torch.zeros(B, cols, dtype=torch.int32)
    return k, table, on_gpu(torch.zeros(B, dtype=torch.int32), index)


def test_page_tables_whose_rows_overlap_are_refused(A):
    """The rows of an expanded table, or of a view that overlaps itself, are not max_pages
    apart; reading them so would pass the table's end."""
    k, table, lens = cache_of()
    for bad in (table[:1].expand(3, 4), torch.zeros(12, dtype=torch.int32).as_strided((3, 4), (2, 1)),
                table[:1, :1].expand(3, 1), torch.zeros(3, 8, dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            A._cache(k, k, on_gpu(bad), lens)
    # rows further apart, and one row whose stride says nothing, are fine
    for good, ld in ((table, 4), (torch.zeros(3, 9, dtype=torch.int32)[:, :4], 9),
                     (table[:, :0], 4)):
        packed, *_ = A._cache(k, k, on_gpu(good), lens)
        assert A._CACHE.unpack(packed)[11] == ld
    one = table[:1].expand(1, 4).as_strided((1, 4), (0, 1))
    packed, *_ = A._cache(k, k, on_gpu(one), on_gpu(torch.zeros(1, dtype=torch.int32)))
    assert A._CACHE.unpack(packed)[11] == 4
