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


@pytest.mark.parametrize("q_heads,kv_heads,dim", [(2, 2, 128), (4, 2, 64), (16, 2, 128), (64, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_of_a_cut_sequence_keep_their_places(lib, ctx, q_heads, kv_heads, dim, causal):
    """Sequence 1 has more rows than the bound says, sequence 2 more tokens, three rows come before the first sequence and five
    behind the last: what is left out gives zeros and -infinity, every other row what the 64-bit rows give at its place."""
    lens, news, most_q, most_kv = [50, 70, 100, 33], [5, 10, 7, 8], 8, 96
    case = R.make_case(43, lens, news, kv_heads, dim, 16, O.CONV_PAPER, fill=0x7F)
    dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, most_q, most_kv)
    dev["q_start"] += 3
    rows = 3 + sum(news) + 5
    q = torch.randn((rows, q_heads, dim), generator=case["g"]).to(torch.bfloat16)
    out = torch.full((rows, q_heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows, q_heads), 7.0, device="cuda")
    ctx.device_flags()
    ctx.attn_paged(cache, batch, q.cuda(), out, causal=causal, lse=lse)
    assert ctx.device_flags() == lib.FLAG_BAD_INDEX
    # one row at a time: a sequence of one new token whose length is what the row sees
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    kept, sees, table = [], [], []
    for b, (length, n) in enumerate(zip(lens, news)):
        for i in range(min(n, most_q)):
            kept.append(3 + sum(news[:b]) + i)
            sees.append(min(length, most_kv, length - n + i + 1 if causal else length))
            table.append(case["table"].numpy()[b])
    want = R.attention(cpu, np.array(table), list(range(len(kept) + 1)), sees, q[kept].double().numpy(), dim ** -0.5, True, O.CONV_PAPER)
    check(out[kept], lse[kept], want)
    left = sorted(set(range(rows)) - set(kept))
    assert (out[left] == 0).all() and torch.isneginf(lse[left]).all()


@pytest.mark.parametrize("news", [1, 30])
def test_more_rows_than_the_sequences_have(lib, ctx, news):
    """A batch padded to a fixed number of rows, with empty sequences at its end: the padding is zeros, nothing else changes."""
    case = R.make_case(44, [40, 300, 0, 0], [news, news, 0, 0], 2, 128, 32, O.CONV_NATIVE)
    dev, cache, batch = gpu_state(lib, case, O.CONV_NATIVE, news, 300)
    q = torch.randn((2 * news + 700, 8, 128), generator=case["g"]).to(torch.bfloat16).cuda()
    want, want_lse = torch.empty_like(q[:2 * news]), torch.empty((2 * news, 8), device="cuda")
    ctx.device_flags()
    ctx.attn_paged(cache, batch, q[:2 * news], want, lse=want_lse)
    assert ctx.device_flags() == 0
    wide = torch.full((q.shape[0], 9, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    ctx.attn_paged(cache, batch, q, wide[:, :8], lse=lse)
    assert ctx.device_flags() == lib.FLAG_BAD_INDEX
    assert torch.equal(wide[:2 * news, :8].contiguous().view(torch.int16), want.view(torch.int16)) and torch.equal(lse[:2 * news], want_lse)
    assert (wide[2 * news:, :8] == 0).all() and torch.isneginf(lse[2 * news:]).all() and (wide[:, 8] == 7.0).all()


def test_append_and_attention_agree_on_a_cut_sequence(lib, ctx):
    """Ten rows under a bound of eight: the rows that enter the cache are the ones that the kept queries see as their own."""
    conv, dim = O.CONV_NATIVE, 64
    for heads in ((2, 2), (16, 2)):
        case = R.make_case(45, [100], [10], heads[1], dim, 16, conv)
        dev, cache, batch = gpu_state(lib, case, conv, 8, 100)
        k, v = (torch.randn((10, heads[1], dim), generator=case["g"]).to(torch.bfloat16).cuda() for _ in range(2))
        q = torch.randn((10, heads[0], dim), generator=case["g"]).to(torch.bfloat16)
        ctx.kv_append(cache, batch, k, v)
        out, lse = torch.empty((10, heads[0], dim), dtype=torch.bfloat16, device="cuda"), torch.empty((10, heads[0]), device="cuda")
        ctx.attn_paged(cache, batch, q.cuda(), out, lse=lse)
        cpu = [dev[n].cpu().numpy() for n in ("k8", "v8", "bk", "bv")]
        own, _ = R.quantise_row(k[7, 0].double().cpu().numpy(), conv)
        assert np.array_equal(R.cached_rows(cpu, case["table"].numpy(), 0, np.array([97]))[0][0, 0], own)
        want = R.attention(cpu, case["table"].numpy(), [0, 10], [100], q.double().numpy(), dim ** -0.5, True, conv)
        check(out[:8], lse[:8], tuple(x[:8] for x in want))
        ctx.device_flags()


def test_calls_that_overlapped_spoil_no_later_call(lib, ctx):
    """Calls of several shapes at the same time on one context are against its contract, and their own outputs are lost.  The
    calls after them, launched or replayed from a graph, give the bits that they gave before."""
    conv, calls = O.CONV_PAPER, []
    for news, heads, lens in ((1, (8, 1), [3000, 1500, 77]), (1, (16, 2), [5000]), (64, (8, 2), [3000, 1500, 77]), (300, (4, 1), [4000])):
        case = R.make_case(46, lens, [news] * len(lens), heads[1], 128, 32, conv)
        dev, cache, batch = gpu_state(lib, case, conv, news, max(lens))
        q = torch.randn((news * len(lens), heads[0], 128), generator=case["g"]).to(torch.bfloat16).cuda()
        calls.append((cache, batch, q))
    own = lib.Context(0)

    def run(i, out=None):
        out = torch.full_like(calls[i][2], float("nan")) if out is None else out
        own.attn_paged(*calls[i], out)
        return out

    want = [run(i) for i in range(len(calls))]
    torch.cuda.synchronize()
    replayed, graphs = [torch.empty_like(w) for w in want], []
    for i in range(len(calls)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(i, replayed[i])
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(5):
        for n in range(40):
            for j, s in enumerate(streams):
                with torch.cuda.stream(s):
                    if j == 0:
                        graphs[n % 4].replay()
                    else:
                        run((n + j) % 4)
        torch.cuda.synchronize()
        for i in range(len(calls)):
            replayed[i].fill_(float("nan"))
            graphs[i].replay()
            assert torch.equal(run(i).view(torch.int16), want[i].view(torch.int16))
            assert torch.equal(replayed[i].view(torch.int16), want[i].view(torch.int16))
    assert own.device_flags() & lib.FLAG_TIMEOUT == 0
    own.close()


def test_attention_goes_on_after_a_wait_ran_out(lib):
    """A wait that runs out (on a barrier that nothing completes, with a limit of 2 ms) and the clearing of its flag, which
    also clears the arrival counters, leave split calls right, launched and replayed."""
    own = lib.Context(0)
    for news, heads in ((1, (8, 1)), (64, (8, 2))):
        case = R.make_case(47, [3000, 1500], [news] * 2, heads[1], 128, 32, O.CONV_PAPER)
        dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, news, 3000)
        q = torch.randn((2 * news, heads[0], 128), generator=case["g"]).to(torch.bfloat16).cuda()
        want, out = torch.empty_like(q), torch.empty_like(q)
        own.attn_paged(cache, batch, q, want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            own.attn_paged(cache, batch, q, out)
        own.selftest_wait_expiry(2_000_000)
        assert own.device_flags(clear=True) & lib.FLAG_TIMEOUT
        for _ in range(3):
            out.fill_(float("nan"))
            graph.replay()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
            again = torch.empty_like(q)
            own.attn_paged(cache, batch, q, again)
            assert torch.equal(again.view(torch.int16), want.view(torch.int16))
        assert own.device_flags() == 0
    own.close()


@pytest.mark.parametrize("news", [1, 2, 40, 150])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gain", [12, 14, 16, 19])
def test_one_query_channel_far_above_the_others(lib, ctx, news, dim, gain):
    """Channel 0 of the queries is 2^gain times the others, and the keys are zero there: the scores come from query numbers far
    below their row's largest.  A query number is held within 2^-21 of the row's largest (exactly, if it is not 2^13 below),
    so to the FP32 sum's 2^-15 of scale * sum |q k| comes 2^-21 of scale * max |q| * sum |k|."""
    lens, heads, kv_heads = [200, 333], 4, 2
    case = R.make_case(48, lens, [news] * 2, kv_heads, dim, 32, O.CONV_PAPER, fill=0x7F)
    case["k8"][..., 0] = 0
    q = torch.randn((2 * news, heads, dim), generator=case["g"])
    q[..., 0] = q[..., 0].sign() * 2.0 ** gain
    q = q.to(torch.bfloat16)
    dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, news, 333)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    ctx.attn_paged(cache, batch, q.cuda(), out, lse=lse)
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    o, l, spread, score = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), dim ** -0.5, True, O.CONV_PAPER)
    for b, n in enumerate(lens):
        kc, kb, _, _ = R.cached_rows(cpu, case["table"].numpy(), b, np.arange(n))
        most = np.abs(R.numbers(kc, kb, O.CONV_PAPER)).sum(-1).max(0).repeat(heads // kv_heads)          # per query head
        rows = slice(b * news, (b + 1) * news)
        score[rows] += 2.0 ** -6 * dim ** -0.5 * np.abs(q[rows].double().numpy()).max(-1) * most
    check(out, lse, (o, l, spread, score))


@pytest.mark.parametrize("news", [1, 40, 150])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gain", [10, 12, 13])
def test_query_numbers_down_to_2_13_below_the_largest_are_exact(lib, ctx, news, dim, gain):
    """Channel 0 is 2^gain, the others lie between 1 and 2 (every mantissa of bf16), the keys are zero in channel 0: nothing is
    lost of the queries, so the scores keep the ordinary bound, 2^-15 of scale * sum |q k| over the channels that count."""
    def edit(case, q):
        case["k8"][..., 0] = 0
        q.copy_(((1 + torch.randint(0, 128, q.shape, generator=case["g"]) / 128.0) * q.float().sign()).to(torch.bfloat16))
        q[..., 0] = 2.0 ** gain
    run_case(lib, ctx, 49, [200, 333], [news] * 2, 4, 2, dim, 32, O.CONV_PAPER, True, edit=edit)


@pytest.mark.parametrize("news", [3, 40, 150])
@pytest.mark.parametrize("causal", [True, False])
def test_queries_that_are_not_finite_and_see_nothing_give_zeros(lib, ctx, news, causal):
    """Rows of empty sequences, and under the causal mask rows before the first cached token, whatever the query holds."""
    def edit(case, q):
        q[0, 1, 3], q[0, 2, 0], q[0, 3, :] = float("inf"), float("nan"), float("-inf")
        q[news, 2, 5] = float("nan")
        q[2 * news:] = float("inf")
    out, lse = run_case(lib, ctx, 50, [0, 2, 0], [news] * 3, 4, 2, 64, 16, O.CONV_PAPER, causal, edit=edit)
    assert (out[:news, :4] == 0).all() and (out[2 * news:, :4] == 0).all() and torch.isneginf(lse[:news]).all()


@pytest.mark.parametrize("news", [1, 2, 40, 150])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("powers", [118, 110, 90, -60, -70])
def test_large_keys_meet_small_queries(lib, ctx, news, dim, powers):
    """Keys of about 2^powers under queries of about 2^-powers: scores of ordinary size, from numbers whose product with the
    other side's normalised row is not an FP32 number."""
    def edit(case, q):
        case["bk"].copy_((case["bk"].int() - powers).clamp(-127, 64).to(torch.int8))
        q.copy_((q.float() * 2.0 ** -powers).to(torch.bfloat16))
    run_case(lib, ctx, 51, [200, 333], [news] * 2, 4, 2, dim, 32, O.CONV_NATIVE, True, edit=edit, fill=0x30)


@pytest.mark.parametrize("news", [1, 40])
def test_a_scale_of_zero_weighs_all_tokens_alike(lib, ctx, news):
    """Also where keys and queries are near the ends of their range."""
    def edit(case, q):
        case["bk"].fill_(-119)
        q.copy_((q.float() * 2.0 ** 120).to(torch.bfloat16))
    run_case(lib, ctx, 52, [200, 333], [news] * 2, 4, 2, 64, 32, O.CONV_NATIVE, True, edit=edit, scale=0.0, fill=0x30)


@pytest.mark.parametrize("news", [1, 40])
@pytest.mark.parametrize("scale", [0.125, -0.125])
def test_keys_of_zeros_under_the_largest_queries(lib, ctx, news, scale):
    def edit(case, q):
        case["k8"][:, :, ::2] = 0
        case["k8"][:, :, 1::2] = 0x80
        q.copy_((q.float().sign() * 3e38).to(torch.bfloat16))
    run_case(lib, ctx, 53, [200, 333], [news] * 2, 4, 2, 64, 32, O.CONV_PAPER, False, edit=edit, scale=scale, fill=0x30)


@pytest.mark.parametrize("news,lens", [(1, [300, 64]), (30, [300, 64]), (150, [300, 200]), (30, [5000, 4000])])
@pytest.mark.parametrize("dim", [64, 128])
def test_equal_weights_are_exact(lib, ctx, news, lens, dim):
    """Queries of zeros: every weight is 1, an output is the mean of its tokens' values.  Nothing but the FP32 sum (2^-20 of the
    mean of |v|, at most 5000 numbers of 4 bits within 2^6 of each other) and the rounding to bf16 is between them."""
    case = R.make_case(54, lens, [news] * 2, 2, dim, 32, O.CONV_NATIVE, fill=0x7F)
    case["bv"].fill_(8)
    case["v8"].copy_(torch.randint(0x28, 0x58, case["v8"].shape, generator=case["g"], dtype=torch.uint8))       # 2^-2 .. 2^4
    dev, cache, batch = gpu_state(lib, case, O.CONV_NATIVE, news, max(lens))
    q = torch.zeros((2 * news, 4, dim), dtype=torch.bfloat16)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    ctx.attn_paged(cache, batch, q.cuda(), out, lse=lse)
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    o, l, spread, _ = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), 1.0, True, O.CONV_NATIVE)
    step = np.exp2(np.floor(np.log2(np.abs(o) * (1 + 2.0 ** -20))) - 7)
    assert (np.abs(out.double().cpu().numpy() - o) <= step / 2 + 2.0 ** -20 * spread).all()
    assert (np.abs(lse.double().cpu().numpy() - l) <= 2.0 ** -19 * (1 + np.abs(l))).all()


@pytest.mark.parametrize("news", [1, 30, 150])
@pytest.mark.parametrize("gain", [0.5, 2.0])
def test_outputs_are_too_large_as_often_as_too_small(lib, ctx, news, gain):
    """Positive values, random scores: the roundings of weights and outputs leave no drift.  An output's rounding to bf16 is
    within 2^-8 of it and evenly spread, 2^-8 / sqrt(12) on average; the mean of n has 1 / sqrt(n) of that, and five times
    as much is allowed, beside 2^-16 for the weights' roundings, which are 2^-11 at most and have either sign."""
    dim, lens = 128, [900, 700, 800, 600]
    case = R.make_case(55, lens, [news] * 4, 4, dim, 32, O.CONV_NATIVE, fill=0x7F)
    case["bv"].fill_(8)
    case["v8"].copy_(torch.randint(0x38, 0x40, case["v8"].shape, generator=case["g"], dtype=torch.uint8))
    q = (torch.randn((4 * news, 16, dim), generator=case["g"]) * gain).to(torch.bfloat16)
    dev, cache, batch = gpu_state(lib, case, O.CONV_NATIVE, news, 900)
    out = torch.empty_like(q, device="cuda")
    ctx.attn_paged(cache, batch, q.cuda(), out)
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    o = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), dim ** -0.5, True, O.CONV_NATIVE)[0]
    drift = (out.double().cpu().numpy() / o - 1).mean()
    assert abs(drift) <= 5 * 2.0 ** -8 / np.sqrt(12 * o.size) + 2.0 ** -16


def large_values(dim, powers, bias, late, everywhere, page=32):
    """Scores of 0 and of about `powers` powers of two, the higher ones on the later tokens (late) or on the earlier; values of the
    tokens with the higher scores, or everywhere, cast under `bias`.  The higher ones hold zeros in the last quarter of
    their dimensions, where the others' weights decide."""
    def edit(case, q):
        q.zero_()
        q[..., 0] = 1.0
        case["k8"].zero_()
        case["bk"].zero_()
        case["bv"].fill_(bias if everywhere else 8)
        for b, n in enumerate(case["kv_len"].tolist()):
            for j in range(n):
                if (j >= n // 2) == late:
                    pg, off = int(case["table"][b, j // page]), j % page
                    case["k8"][pg, :, off, 0] = 0x38 - j % 2
                    case["bv"][pg, :, off] = bias
                    if powers <= 55:
                        case["v8"][pg, :, off, 3 * dim // 4:] = 0
    return edit


@pytest.mark.parametrize("news,heads", [(1, (8, 1)), (2, (8, 1)), (40, (4, 2)), (150, (4, 2))])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("powers", [0, 30, 39.5, 50, 59, 90])
@pytest.mark.parametrize("bias", [-42, -72, -119])
def test_large_values_stay_finite(lib, ctx, news, heads, dim, powers, bias):
    """Values up to 3e38 under weights that differ by up to 2^90: where the result is a finite number, so is the output."""
    lens = [200, 333]
    for late in (True, False):
        for everywhere in (False, True):
            run_case(lib, ctx, 56, lens, [news] * 2, heads[0], heads[1], dim, 32, O.CONV_NATIVE, True, scale=powers * float(np.log(2)),
                     edit=large_values(dim, powers, bias, late, everywhere))


@pytest.mark.parametrize("news,heads", [(1, (8, 1)), (40, (4, 1))])
def test_large_values_in_long_contexts(lib, ctx, news, heads):
    """... also where a context is split: some parts hold large values, others none."""
    for powers, late in ((0, True), (39.5, True), (50, False)):
        run_case(lib, ctx, 57, [6000], [news], heads[0], heads[1], 128, 64, O.CONV_NATIVE, True, scale=powers * float(np.log(2)),
                 edit=large_values(128, powers, -119, late, powers == 0, page=64))


@pytest.mark.parametrize("news", [1, 40])
def test_stale_biases_change_nothing(lib, ctx, news):
    """Biases of large values behind a sequence's end, in its own pages: the same bits as with other bytes there."""
    outs = []
    for stale in (8, -119):
        case = R.make_case(58, [201, 333], [news] * 2, 2, 128, 128, O.CONV_NATIVE, fill=0x30)
        held = case["bv"] != -128
        case["bv"][~held] = stale
        dev, cache, batch = gpu_state(lib, case, O.CONV_NATIVE, news, 333)
        q = torch.randn((2 * news, 8, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        ctx.attn_paged(cache, batch, q, out, lse=lse)
        outs.append((out, lse))
    assert torch.equal(outs[0][0].view(torch.int16), outs[1][0].view(torch.int16)) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("news", [1, 40])
def test_a_cache_beyond_32_bits(lib, ctx, news):
    """A cache of 4.6 GB whose keys and values of a page share one buffer; the tokens lie in its first and its last pages."""
    pages, heads, size, dim, conv = 70000, 2, 128, 128, O.CONV_NATIVE
    lens = [300, 170]
    case = R.make_case(59, lens, [news] * 2, heads, dim, size, conv)
    both = torch.zeros((pages, 2, heads, size, dim), dtype=torch.uint8, device="cuda")
    biases = torch.zeros((pages, 2, heads, size), dtype=torch.int8, device="cuda")
    assert both.numel() > 1 << 32
    far = torch.tensor([0, pages - 1, 35001, pages - 2, 1, pages - 3, 2, pages - 4])[:case["k8"].shape[0]]
    for n, part, t in (("k8", 0, both), ("v8", 1, both), ("bk", 0, biases), ("bv", 1, biases)):
        t[far.cuda(), part] = case[n].cuda()
    cache = lib.KvCache(both[:, 0], both[:, 1], biases[:, 0], biases[:, 1], conv=conv)
    batch = lib.SeqBatch(case["q_start"].cuda(), case["kv_len"].cuda(), far[case["table"].long()].to(torch.int32).cuda(), news, 300)
    q = torch.randn((2 * news, 8, dim), generator=case["g"]).to(torch.bfloat16)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    ctx.attn_paged(cache, batch, q.cuda(), out, lse=lse)
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    check(out, lse, R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), dim ** -0.5, True, conv))


@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 1, 128), (4, 4, 64), (32, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_a_chunk_beside_many_single_tokens(lib, ctx, q_heads, kv_heads, dim, causal):
    """What a step of a server that takes in a prompt while others go on looks like: units of one row and of 256 alternate."""
    lens = [3, 700, 64, 129, 1, 300, 515] * 5 + [600]
    news = [1] * 35 + [290]
    lens[17], news[17], lens[3], news[3] = 400, 130, 0, 0
    run_case(lib, ctx, 60, lens, news, q_heads, kv_heads, dim, 32, O.CONV_PAPER, causal)
