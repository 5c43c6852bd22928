"""Attention over the paged FP8 cache (fp8_attn_paged) against a plain 64-bit implementation on the same bytes.

Bounds, derived from how the kernels round:
  output: one rounding to bf16 (half the distance between bf16 numbers there), the softmax numerators held in at least 11 bits before they meet the values
  (2^-11, doubled for the statistics: 2^-10 of sum p|v| / sum p) and the scores' own error, an FP32 sum of head_dim
  products whose query factor is exact to 2^-17 of the row's largest: e = 2^-15 of the largest scale * sum |q k|, which
  moves numerators and denominator by up to e each (2 e of the same spread).
  lse: e, and FP32 statistics (2^-19 of 1 + |lse|).
"""
import numpy as np
import pytest
import torch

import kv_reference as R
import oracle as O

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


def gpu_state(lib, case, conv, max_q, max_kv):
    dev = {n: case[n].cuda() for n in ("k8", "v8", "bk", "bv", "table", "q_start", "kv_len")}
    cache = lib.KvCache(dev["k8"], dev["v8"], dev["bk"], dev["bv"], conv=conv)
    batch = lib.SeqBatch(dev["q_start"], dev["kv_len"], dev["table"], max_q_len=max_q, max_kv_len=max_kv)
    return dev, cache, batch


def check(out, lse, want, what=""):
    o, l, spread, score = want
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    e = score * 2.0 ** -15
    nan = np.isnan(o)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    before = spread * (2.0 ** -10 + 2 * e[..., None])             # what the rounding to bf16 is applied to
    step = np.exp2(np.floor(np.log2(np.abs(o) + before + 2.0 ** -126)) - 7)
    tol = before + step / 2
    bad = (np.abs(got - o) > tol) & ~nan
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outputs off, first at {np.argwhere(bad)[0]}: got {got[bad][0]}, want {o[bad][0]} +- {tol[bad][0]}"
    fin = np.isfinite(l)
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(l)) and np.array_equal(np.isnan(got_lse), np.isnan(l)), what
    off = np.abs(got_lse[fin] - l[fin]) > e[fin] + 2.0 ** -19 * (1 + np.abs(l[fin]))
    assert not off.any(), f"{what}: {off.sum()} lse values off"


def run_case(lib, ctx, seed, lens, news, q_heads, kv_heads, dim, page, conv, causal, fill=0x7F, q_gain=1.0, edit=None, scale=None):
    case = R.make_case(seed, lens, news, kv_heads, dim, page, conv, fill=fill)
    T = sum(news)
    q = (torch.randn((T, q_heads + 2, dim), generator=case["g"]) * q_gain).to(torch.bfloat16)
    if edit:
        edit(case, q)
    dev, cache, batch = gpu_state(lib, case, conv, max(1, max(news)), max(1, max(lens)))
    qd = q.cuda()[:, 1:1 + q_heads]
    out = torch.full((T, q_heads + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, q_heads), 7.0, device="cuda")
    ctx.device_flags()
    ctx.attn_paged(cache, batch, qd, out[:, :q_heads], causal=causal, lse=lse, scale=scale)
    flags = ctx.device_flags()
    assert flags & (lib.FLAG_TIMEOUT | lib.FLAG_BAD_INDEX) == 0
    assert (out[:, q_heads:] == 7.0).all()
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    want = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), case["kv_len"].numpy(),
                       q[:, 1:1 + q_heads].double().numpy(), dim ** -0.5 if scale is None else scale, causal, conv)
    check(out[:, :q_heads], lse, want, f"lens {lens} news {news}")
    # without the second output: the same bits
    again = torch.empty((T, q_heads, dim), dtype=torch.bfloat16, device="cuda")
    ctx.attn_paged(cache, batch, qd, again, causal=causal, scale=scale)
    assert torch.equal(again.view(torch.int16), out[:, :q_heads].contiguous().view(torch.int16))
    return out, lse


HEADS = [(8, 1), (8, 8), (6, 2), (10, 2), (32, 1), (3, 3)]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads,kv_heads", HEADS)
def test_single_tokens(lib, ctx, page, dim, q_heads, kv_heads):
    lens = [1, 2, 15, 16, 17, 100, 128, 129, 260, 511]
    run_case(lib, ctx, 21, lens, [1] * len(lens), q_heads, kv_heads, dim, page, O.CONV_PAPER, True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("q_heads,kv_heads", [(8, 1), (4, 4), (10, 2)])
def test_a_few_tokens(lib, ctx, causal, dim, page, q_heads, kv_heads):
    lens, news = [2, 9, 40, 130, 257, 3, 16], [2, 3, 1, 5, 2, 3, 0]
    run_case(lib, ctx, 22, lens, news, q_heads, kv_heads, dim, page, O.CONV_NATIVE, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 128), (128, 16), (64, 64), (128, 32)])
@pytest.mark.parametrize("q_heads,kv_heads", [(8, 1), (2, 2), (5, 1)])
def test_chunks(lib, ctx, causal, dim, page, q_heads, kv_heads):
    lens, news = [129, 300, 65, 513, 128], [129, 33, 64, 150, 1]
    run_case(lib, ctx, 23, lens, news, q_heads, kv_heads, dim, page, O.CONV_PAPER, causal)


@pytest.mark.parametrize("news", [[1, 1, 1, 1], [5, 2, 4, 1], [40, 20, 60, 33]])
def test_rows_without_a_token_give_zeros(lib, ctx, news):
    """Empty sequences, and more new rows than cached tokens under the causal mask."""
    for causal in (True, False):
        out, lse = run_case(lib, ctx, 24, [0, 1, 3, 30], news, 4, 2, 128, 16, O.CONV_PAPER, causal)
        assert (out[:news[0], :4] == 0).all() and torch.isneginf(lse[:news[0]]).all()


@pytest.mark.parametrize("rows", [1, 3, 70])
def test_special_numbers_reach_only_the_rows_that_see_them(lib, ctx, rows):
    """A row marked non-finite poisons the queries that see it and no other; NaN bytes behind a sequence's end, in its
    own pages and in others', reach nobody (every case here is filled with them)."""
    def edit(case, q):
        page = int(case["table"][1, 2])
        case["bv"][page, 0, 3] = -128                       # token 35 of sequence 1
        case["v8"][page, 0, 3, 5] = 0x7F
        page = int(case["table"][2, 0])
        case["bk"][page, 1, 9] = -128
        case["k8"][page, 1, 9, :] = 0xFF
        q[0, 1, 3] = float("inf")
        q[1, 2, 0] = float("nan")
    lens = [90, 36 + 1, 100]
    run_case(lib, ctx, 25, lens, [rows, min(rows, 37), rows], 4, 2, 128, 16, O.CONV_PAPER, True, edit=edit)


@pytest.mark.parametrize("news", [1, 2, 50])
@pytest.mark.parametrize("dim", [64, 128])
def test_numbers_of_very_different_size(lib, ctx, news, dim):
    """Scores up to a few hundred (one key takes all), value rows whose magnitudes differ by 2^40, queries of 2^-30."""
    def edit(case, q):
        g = case["g"]
        case["bv"].copy_(torch.randint(-18, 22, case["bv"].shape, generator=g, dtype=torch.int8))
        case["bk"].copy_(torch.randint(4, 12, case["bk"].shape, generator=g, dtype=torch.int8))
        q[:, 2] *= 2.0 ** -30
        q[:, 3, 1:] *= 2.0 ** -12
    run_case(lib, ctx, 26, [200, 300], [news, news], 4, 2, dim, 32, O.CONV_PAPER, True, q_gain=4.0, edit=edit, fill=0x7E)


def test_scale_argument(lib, ctx):
    for news in (1, 40):
        run_case(lib, ctx, 27, [150, 70], [news, news], 8, 2, 64, 16, O.CONV_NATIVE, True, scale=0.011)
        run_case(lib, ctx, 27, [150, 70], [news, news], 8, 2, 64, 16, O.CONV_NATIVE, False, scale=-0.05)
        run_case(lib, ctx, 27, [150, 70], [news, news], 8, 2, 64, 16, O.CONV_NATIVE, False, scale=0.0)


@pytest.mark.parametrize("news,q_heads,kv_heads", [(1, 8, 1), (1, 2, 2), (9, 8, 1), (200, 8, 1)])
def test_long_contexts_are_split_and_joined(lib, ctx, news, q_heads, kv_heads):
    run_case(lib, ctx, 28, [9000, 4111], [news, news], q_heads, kv_heads, 128, 64, O.CONV_PAPER, True)


def test_many_short_sequences(lib, ctx):
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 60, 700)]
    for most in (1, 4):
        news = [int(x) for x in rng.integers(0, most + 1, 700)]
        run_case(lib, ctx, 29, lens, news, 4, 1, 64, 16, O.CONV_PAPER, True)


def test_repeated_calls_give_the_same_bits_on_a_busy_gpu_and_on_another_stream(lib, ctx):
    for news, heads in ((1, (8, 1)), (64, (8, 2))):
        case = R.make_case(30, [3000, 1500, 77], [news] * 3, heads[1], 128, 32, O.CONV_PAPER)
        dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, news, 3000)
        q = torch.randn((3 * news, heads[0], 128), generator=case["g"]).to(torch.bfloat16).cuda()
        first = torch.empty_like(q)
        ctx.attn_paged(cache, batch, q, first)
        torch.cuda.synchronize()
        busy, own = torch.cuda.Stream(), torch.cuda.Stream()
        a = torch.randn((2048, 2048), device="cuda")
        with torch.cuda.stream(busy):
            for _ in range(30):
                a = a @ a * 1e-3
        with torch.cuda.stream(own):
            outs = [torch.full_like(q, float("nan")) for _ in range(20)]
            for o in outs:
                ctx.attn_paged(cache, batch, q, o)
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("q_heads,kv_heads,dim", [(32, 32, 64), (8, 8, 128), (16, 2, 128)])
def test_units_of_one_step_and_of_several_follow_one_another(lib, ctx, q_heads, kv_heads, dim):
    """Contexts whose lengths leave one step of a (sequence, head) to a multiprocessor before or behind several of the
    next, in calls that nothing waits between: what one unit leaves behind must not reach the next."""
    lens, news = [701, 543, 595, 492, 461, 90, 128, 300], [37, 23, 23, 19, 30, 33, 17, 30]
    case = R.make_case(34, lens, news, kv_heads, dim, 16, O.CONV_NATIVE, fill=0x7F)
    dev, cache, batch = gpu_state(lib, case, O.CONV_NATIVE, 37, 701)
    q = torch.randn((sum(news), q_heads, dim), generator=case["g"]).to(torch.bfloat16)
    qd = q.cuda()
    outs = [(torch.empty_like(qd), torch.empty(qd.shape[:2], device="cuda")) for _ in range(30)]
    for o, l in outs:
        ctx.attn_paged(cache, batch, qd, o, lse=l)
    torch.cuda.synchronize()
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    want = R.attention(cpu, case["table"].numpy(), case["q_start"].numpy(), lens, q.double().numpy(), dim ** -0.5, True, O.CONV_NATIVE)
    check(*outs[0], want)
    for o, l in outs[1:]:
        assert torch.equal(o.view(torch.int16), outs[0][0].view(torch.int16)) and torch.equal(l, outs[0][1])


def test_launches_are_counted(lib, ctx):
    for news in (1, 40):
        case = R.make_case(35, [200, 90], [news] * 2, 2, 64, 16, O.CONV_PAPER)
        dev, cache, batch = gpu_state(lib, case, O.CONV_PAPER, news, 200)
        q = torch.zeros((2 * news, 4, 64), dtype=torch.bfloat16, device="cuda")
        k = torch.zeros((2 * news, 2, 64), dtype=torch.bfloat16, device="cuda")
        before = lib.launch_count()
        ctx.kv_append(cache, batch, k, k)
        ctx.attn_paged(cache, batch, q, torch.empty_like(q))
        ctx.kv_read(cache, batch, k, None)
        assert lib.launch_count() == before + 3


def test_graph_replay_follows_the_lengths_on_the_device(lib, ctx):
    """Captured once; the lengths, the tokens and the pages of later replays come from device memory."""
    conv, heads, dim = O.CONV_PAPER, 2, 128
    case = R.make_case(31, [300, 300], [1, 1], heads, dim, 16, conv)
    dev, cache, batch = gpu_state(lib, case, conv, 1, 300)
    q = torch.randn((2, 8, dim), generator=case["g"]).to(torch.bfloat16).cuda()
    k, v = (torch.randn((2, heads, dim), generator=case["g"]).to(torch.bfloat16).cuda() for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx.kv_append(cache, batch, k, v)
        ctx.attn_paged(cache, batch, q, out, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.kv_append(cache, batch, k, v)
        ctx.attn_paged(cache, batch, q, out, lse=lse)
    for lens in ([300, 17], [1, 299], [44, 160]):
        dev["kv_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        cpu = [dev[n].cpu().numpy() for n in ("k8", "v8", "bk", "bv")]
        want = R.attention(cpu, case["table"].numpy(), [0, 1, 2], lens, q.double().cpu().numpy(), dim ** -0.5, True, conv)
        check(out, lse, want, str(lens))


def test_pages_and_lengths_out_of_bounds_are_flagged(lib, ctx):
    conv = O.CONV_PAPER
    for news in (1, 60):
        case = R.make_case(32, [100, 100, 100], [news] * 3, 2, 128, 16, conv)
        case["table"][1, 3] = 1 << 20
        case["kv_len"][2] = 5000
        dev, cache, batch = gpu_state(lib, case, conv, news, 100)
        q = torch.randn((3 * news, 4, 128), generator=case["g"]).to(torch.bfloat16).cuda()
        out = torch.zeros_like(q)
        ctx.device_flags()
        ctx.attn_paged(cache, batch, q, out)
        assert ctx.device_flags() & lib.FLAG_BAD_INDEX
        assert not torch.isnan(out[:news]).any() and torch.isnan(out[2 * news - 1]).all()


def test_refusals(lib, ctx):
    conv = O.CONV_PAPER
    case = R.make_case(33, [20], [4], 2, 64, 16, conv)
    dev, cache, batch = gpu_state(lib, case, conv, 4, 20)
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    batch._desc.tokens = 4
    fn = lib.raw().fp8_attn_paged

    def status(qp=q.data_ptr(), ld_q=256, heads=4, op=out.data_ptr(), ld_o=256, lse=None, scale=0.1, conv=conv, h=ctx._h):
        return fn(h, cache._ref, batch._ref, qp, ld_q, heads, op, ld_o, lse, scale, 1, conv, None)

    assert status() == lib.OK
    assert status(qp=None) == status(op=None) == status(h=None) == lib.ERR_NULL
    assert status(heads=0) == status(heads=3) == status(heads=8) == status(ld_q=248) == status(ld_o=255) == lib.ERR_SHAPE
    assert status(scale=float("nan")) == status(scale=float("inf")) == lib.ERR_SHAPE
    assert status(qp=q.data_ptr() + 8) == status(ld_q=260) == status(op=out.data_ptr() + 2) == status(ld_o=257) == lib.ERR_ALIGN
    assert status(lse=out.data_ptr() + 2) == lib.ERR_ALIGN
    assert status(conv=5) == lib.ERR_DTYPE
    with pytest.raises(ValueError):
        ctx.attn_paged(cache, batch, q.float(), out)
    with pytest.raises(ValueError):
        ctx.attn_paged(cache, batch, q, out[:, :, ::2])
    with pytest.raises(ValueError):
        ctx.attn_paged(cache, batch, q, out, lse=torch.zeros((4, 5), device="cuda"))
