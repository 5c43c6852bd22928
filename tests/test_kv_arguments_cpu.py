"""Arguments of the cache calls that are refused before a pointer reaches the library (no GPU: the tensors only claim to be
on one, and the context has no handle)."""
import pytest
import torch

from paper_2309_17224_b200 import build as B

B.build()
from paper_2309_17224_b200 import fp8lin


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_gpu(t):
    return t.as_subclass(OnGpu)


def zeros(*shape, dtype=torch.bfloat16):
    return on_gpu(torch.zeros(shape, dtype=dtype))


@pytest.fixture
def ctx():
    c = object.__new__(fp8lin.Context)
    c._h, c.device = None, 0
    return c


def cache_of(pages=8, heads=2, size=16, dim=64):
    k8, v8 = (zeros(pages, heads, size, dim, dtype=torch.uint8) for _ in range(2))
    bk, bv = (zeros(pages, heads, size, dtype=torch.int8) for _ in range(2))
    return fp8lin.KvCache(k8, v8, bk, bv)


def batch_of(table, max_kv_len, seqs=2):
    return fp8lin.SeqBatch(zeros(seqs + 1, dtype=torch.int32), zeros(seqs, dtype=torch.int32), table, max_q_len=4,
                           max_kv_len=max_kv_len)


def calls(ctx, cache, batch):
    rows, q = zeros(4, 2, 64), zeros(4, 4, 64)
    return [lambda: ctx.kv_append(cache, batch, rows, rows), lambda: ctx.kv_read(cache, batch, rows, None),
            lambda: ctx.attn_paged(cache, batch, q, q)]


def test_a_table_slice_with_too_few_columns_is_refused(ctx):
    """Two columns of a table that is eight wide: the rows lie far enough apart for 64 tokens, but hold 32."""
    wide = zeros(2, 8, dtype=torch.int32)
    for call in calls(ctx, cache_of(), batch_of(wide[:, 6:], 33)):
        with pytest.raises(ValueError, match="columns"):
            call()
    for call in calls(ctx, cache_of(), batch_of(wide[:1, :2], 33, seqs=1)):
        with pytest.raises(ValueError, match="columns"):
            call()


def test_lengths_are_one_per_sequence():
    with pytest.raises(ValueError):
        fp8lin.SeqBatch(zeros(3, dtype=torch.int32), zeros(2, 2, dtype=torch.int32), zeros(2, 8, dtype=torch.int32), 4, 33)


def test_tensors_in_host_memory_are_refused(ctx):
    cache, batch = cache_of(), batch_of(zeros(2, 8, dtype=torch.int32), 33)
    rows, q = zeros(4, 2, 64), zeros(4, 4, 64)
    host, host_q = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    lse = torch.zeros((4, 4))
    for call in (lambda: ctx.kv_append(cache, batch, host, rows), lambda: ctx.kv_append(cache, batch, rows, host),
                 lambda: ctx.kv_read(cache, batch, None, host), lambda: ctx.attn_paged(cache, batch, host_q, q),
                 lambda: ctx.attn_paged(cache, batch, q, host_q), lambda: ctx.attn_paged(cache, batch, q, q, lse=lse)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_other_types_and_shapes_are_refused(ctx):
    cache, batch = cache_of(), batch_of(zeros(2, 8, dtype=torch.int32), 33)
    rows = zeros(4, 2, 64, dtype=torch.float64)
    with pytest.raises(ValueError, match="bf16, fp16 or fp32"):
        ctx.kv_append(cache, batch, rows, rows)
    with pytest.raises(ValueError):
        ctx.attn_paged(cache, batch, zeros(256), zeros(256))


def test_handles_of_another_gpu_are_refused(ctx):
    ctx.device = 1
    for call in calls(ctx, cache_of(), batch_of(zeros(2, 8, dtype=torch.int32), 33)):
        with pytest.raises(ValueError, match="GPU 1"):
            call()


def test_calls_leave_a_shared_batch_as_it_is(ctx, monkeypatch):
    """Two threads on one batch: a call sees its own number of rows, whatever another call sets in between."""
    cache, batch = cache_of(), batch_of(zeros(2, 8, dtype=torch.int32), 33)
    before, seen = bytes(batch._desc), []

    def library(h, cache_ref, batch_ref, *rest):
        seen.append((batch_ref._obj.tokens, batch_ref._obj.seqs, batch_ref._obj.max_kv_len))
        if len(seen) == 1:                                        # a call of another thread, before this one reads
            ctx.kv_append(cache, batch, zeros(7, 2, 64), zeros(7, 2, 64))
            seen.append((batch_ref._obj.tokens, batch_ref._obj.seqs, batch_ref._obj.max_kv_len))
        return fp8lin.OK

    monkeypatch.setattr(fp8lin._lib, "fp8_kv_append", library)
    monkeypatch.setattr(fp8lin, "_raw_stream", lambda device: None)
    ctx.kv_append(cache, batch, zeros(4, 2, 64), zeros(4, 2, 64))
    assert seen == [(4, 2, 33), (7, 2, 33), (4, 2, 33)]
    assert bytes(batch._desc) == before


def test_calls_without_rows_launch_nothing(ctx, monkeypatch):
    def library(*args):
        raise AssertionError("called")
    for name in ("fp8_kv_append", "fp8_kv_read", "fp8_attn_paged"):
        monkeypatch.setattr(fp8lin._lib, name, library)
    cache, batch = cache_of(), batch_of(zeros(2, 8, dtype=torch.int32), 33)
    rows, q = zeros(0, 2, 64), zeros(0, 4, 64)
    ctx.kv_append(cache, batch, rows, rows)
    ctx.kv_read(cache, batch, rows, None)
    ctx.attn_paged(cache, batch, q, q)
    with pytest.raises(ValueError):
        ctx.attn_paged(cache, batch, q, zeros(1, 4, 64))


def test_a_pool_makes_batches_without_rows(monkeypatch):
    from paper_2309_17224_b200 import serving
    make = torch.tensor
    monkeypatch.setattr(serving.torch, "tensor", lambda data, dtype, device: on_gpu(make(data, dtype=dtype)))
    pool = serving.PagePool(4, 16)
    pool.extend(["a", "b"], [20, 0])
    for seqs in (["a"], ["a", "b"], []):
        batch = pool.batch(seqs, [0] * len(seqs))
        assert batch.q_start.tolist() == [0] * (len(seqs) + 1) and batch.page_table.shape[0] == len(seqs)
