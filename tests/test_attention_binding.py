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


class Library:
    """Records the calls, and the device that was current at each."""

    def __init__(self, current):
        self.calls, self.current = [], current

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current[0], args[-1]))
            return 0
        return call


@pytest.fixture
def two_gpus(A, monkeypatch):
    """GPU 0 is current; the stream of GPU i is 100 + i."""
    current = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *exc):
            current[0] = self.before

    library = Library(current)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(A, "_current_device", lambda: current[0])
    monkeypatch.setattr(A, "_raw_stream", lambda dev: 100 + dev)
    monkeypatch.setattr(A._sls, "_lib", library)
    monkeypatch.setattr(A._sls, "_CHECK_STATUS", False)
    monkeypatch.setattr(A, "_decode_bytes", lambda *a: 512)
    monkeypatch.setattr(A, "_prefill_bytes", lambda *a: 512)
    return library


def tensors(index):
    k, table, lens = cache_of(index=index)
    q = on_gpu(torch.zeros(3, 4, 64, dtype=torch.bfloat16), index)
    kv = on_gpu(torch.zeros(3, 2, 64, dtype=torch.bfloat16), index)
    cu = on_gpu(torch.arange(4, dtype=torch.int32), index)
    return q, kv, (k, k, on_gpu(table, index), lens), cu


@pytest.mark.parametrize("index", [0, 1])
def test_calls_run_on_the_tensors_device(A, two_gpus, index):
    q, kv, cache, cu = tensors(index)
    ws = on_gpu(torch.zeros(1024, dtype=torch.uint8), index)
    A.qkv_append(q, kv, kv, *cache, out=q)
    A.attention_prefill(q, *cache, cu, workspace=ws, out=q)
    A.attention_decode(q, *cache, workspace=ws, out=q)
    assert two_gpus.calls == [(name, index, 100 + index) for name in (
        "sls_qkv_append", "sls_attention_prefill", "sls_attention_decode")]
    assert two_gpus.current == [0]


def test_what_lies_on_another_gpu_is_refused(A, two_gpus):
    q, kv, cache, cu = tensors(1)
    rope = A.Rope(on_gpu(torch.zeros(32), 0))
    with pytest.raises(ValueError, match="rope"):
        A.qkv_append(q, kv, kv, *cache, rope=rope, out=q)
    for ws in (on_gpu(torch.zeros(1024, dtype=torch.uint8), 0), torch.zeros(1024, dtype=torch.uint8),
               on_gpu(torch.zeros(1024), 1), on_gpu(torch.zeros(2048, dtype=torch.uint8)[::2], 1),
               on_gpu(torch.zeros(1, dtype=torch.uint8).expand(1024), 1)):
        for call in (lambda: A.attention_prefill(q, *cache, cu, workspace=ws, out=q),
                     lambda: A.attention_decode(q, *cache, workspace=ws, out=q)):
            with pytest.raises(ValueError, match="workspace"):
                call()
    other = on_gpu(torch.zeros(3, 4, 64, dtype=torch.bfloat16), 0)
    with pytest.raises(ValueError):
        A.attention_decode(other, *cache, out=other)
    assert two_gpus.calls == []
