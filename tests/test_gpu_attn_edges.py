"""Attention over the paged FP8 cache at its edges: products that follow one another in tensor memory, sequences beyond
their bounds, numbers near the ends of the range.  Bounds as in test_gpu_attn.py unless a test derives its own."""
import numpy as np
import pytest
import torch

import kv_reference as R
import oracle as O
from test_gpu_attn import check, gpu_state, run_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads,kv_heads", [(64, 8), (8, 1)])
def test_units_of_two_tiles_and_of_one_share_the_columns_in_turn(lib, ctx, dim, q_heads, kv_heads):
    """384 and 200 rows a head: units of two query tiles, of one full and of one part tile follow one another, so scores are
    written to the columns that weights of the unit before lie in.  Raw scores are 2^10 and more times the weights: one
    that took a weight's place too early shows."""
    lens, news = [1000, 777, 130, 513, 300], [48, 25, 48, 33, 48]
    case = R.make_case(41, lens, news, kv_heads, dim, 32, O.CONV_PAPER, fill=0x7F)
    dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, 48, 1000)
    q = torch.randn((sum(news), q_heads, dim), generator=case["g"]).to(torch.bfloat16)
    qd = q.cuda()
    busy = torch.cuda.Stream()
    a = torch.empty(192 << 20, dtype=torch.uint8, device="cuda")
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    outs = [(torch.empty_like(qd), torch.empty(qd.shape[:2], device="cuda")) for _ in range(30)]
    for n, (o, l) in enumerate(outs):
        if n % 3 == 0:
            with torch.cuda.stream(busy):
                b.copy_(a)
        ctx.attn_paged(cache, batch, qd, o, lse=l)
    torch.cuda.synchronize()
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    want = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), dim ** -0.5, True, O.CONV_PAPER)
    check(*outs[0], want)
    for o, l in outs[1:]:
        assert torch.equal(o.view(torch.int16), outs[0][0].view(torch.int16)) and torch.equal(l, outs[0][1])


@pytest.mark.parametrize("news", [1, 40])
@pytest.mark.parametrize("bound", [2 ** 31 - 1, 2 ** 31 - 100, 2 ** 30])
def test_the_largest_length_bounds(lib, ctx, news, bound):
    """A bound that says nothing (one sequence, so its table needs no second row) gives what a tight one gives."""
    case = R.make_case(42, [90], [news], 2, 64, 16, O.CONV_PAPER)
    dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, news, 90)
    q = torch.randn((news, 8, 64), generator=case["g"]).to(torch.bfloat16).cuda()
    want, out = torch.empty_like(q), torch.zeros_like(q)
    ctx.attn_paged(cache, batch, q, want)
    desc = type(batch._desc).from_buffer_copy(batch._desc)
    desc.tokens, desc.max_kv_len, desc.table_stride = news, bound, 1 << 27
    ctx.device_flags()
    status = lib.raw().fp8_attn_paged(ctx._h, cache._ref, lib.byref(desc), q.data_ptr(), 512, 8, out.data_ptr(), 512, None,
                                      64 ** -0.5, 1, cache.conv, None)
    torch.cuda.synchronize()
    assert status == lib.OK and ctx.device_flags() == 0
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -10)
