"""The paged FP8 key/value cache: quantising rows as they are written and reading them back (fp8_kv_append, fp8_kv_read).

Bytes and biases are held to a plain 64-bit implementation bit for bit, numbers read back likewise (one rounding to the
output type); every byte that no new token owns must stay as it was.
"""
import numpy as np
import pytest
import torch

import kv_reference as R
import oracle as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context(0)
    yield c
    c.close()


def on_gpu(lib, case, conv, max_q, max_kv):
    dev = {n: case[n].cuda() for n in ("k8", "v8", "bk", "bv", "table", "q_start", "kv_len")}
    cache = lib.KvCache(dev["k8"], dev["v8"], dev["bk"], dev["bv"], conv=conv)
    batch = lib.SeqBatch(dev["q_start"], dev["kv_len"], dev["table"], max_q_len=max_q, max_kv_len=max_kv)
    return dev, cache, batch


def expected_append(case, k, v, conv):
    want = {n: case[n].numpy().copy() for n in ("k8", "v8", "bk", "bv")}
    page = want["k8"].shape[2]
    qs, lens, table = case["q_start"].numpy(), case["kv_len"].numpy(), case["table"].numpy()
    for b in range(len(lens)):
        n = qs[b + 1] - qs[b]
        for i in range(n):
            pos = lens[b] - n + i
            if pos < 0:
                continue
            pg, off = table[b, pos // page], pos % page
            for x, codes, bias in ((k, "k8", "bk"), (v, "v8", "bv")):
                for h in range(x.shape[1]):
                    want[codes][pg, h, off], want[bias][pg, h, off] = R.quantise_row(x[qs[b] + i, h], conv)
    return want


def compare_cache(dev, want):
    for n in ("k8", "v8"):
        got = dev[n].cpu().numpy()
        nan = (want[n] & 127) == 127
        assert np.array_equal((got & 127) == 127, nan)
        assert np.array_equal(got[~nan], want[n][~nan])
    for n in ("bk", "bv"):
        assert np.array_equal(dev[n].cpu().numpy(), want[n])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,page,conv", [(1, 16, O.CONV_PAPER), (3, 32, O.CONV_NATIVE), (8, 128, O.CONV_PAPER), (5, 64, O.CONV_NATIVE)])
def test_append_matches_the_64_bit_rows(lib, ctx, dim, dtype, heads, page, conv):
    lens, news = [37, 1, 0, 131, 16, 5], [21, 1, 0, 64, 0, 9]    # the last has more rows than tokens: four are left out
    case = R.make_case(11, lens, news, heads, dim, page, conv)
    T = sum(news)
    # K and V as columns of a wider matrix, as a QKV matmul leaves them
    wide = torch.randn((T, (2 * heads + 1) * dim), generator=case["g"]) * torch.exp2(torch.randint(-9, 9, (T, 1), generator=case["g"]).float())
    wide = wide.to(DT[dtype]).cuda()
    k = wide[:, dim:(heads + 1) * dim].unflatten(1, (heads, dim))
    v = wide[:, (heads + 1) * dim:].unflatten(1, (heads, dim))
    dev, cache, batch = on_gpu(lib, case, conv, 64, 131)
    ctx.device_flags()
    ctx.kv_append(cache, batch, k, v)
    compare_cache(dev, expected_append(case, k.double().cpu().numpy(), v.double().cpu().numpy(), conv))
    assert ctx.device_flags() & lib.FLAG_BAD_INDEX == 0


def test_reference_rows_agree_with_the_oracle():
    rng = np.random.default_rng(3)
    for conv in (O.CONV_PAPER, O.CONV_NATIVE):
        for _ in range(40):
            x = (rng.standard_normal(64) * 2.0 ** rng.integers(-12, 12)).astype(np.float32)
            bits = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
            _, bias, codes = O.quantise(bits.reshape(1, -1), O.E4, conv)
            got, stored = R.quantise_row((bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64), conv)
            assert stored == bias and np.array_equal(got, codes.reshape(-1))


@pytest.mark.parametrize("conv", [O.CONV_PAPER, O.CONV_NATIVE])
def test_special_rows(lib, ctx, conv):
    D, rows = 64, []
    base = torch.linspace(-1, 1, D)
    rows.append((base * 0, lib.FLAG_ZERO_AMAX))
    for at, val in ((3, float("inf")), (63, float("-inf")), (0, float("nan"))):
        r = base.clone(); r[at] = val
        rows.append((r, lib.FLAG_NONFINITE_AMAX))
    rows.append((base * 2.0 ** -58, 0))            # limited bias
    rows.append((base * 2.0 ** -100, 0))           # every number flushes or lands among the subnormals
    rows.append((base * 3e38, 0))
    rows.append((base * 1e-42, 0))
    rows.append((base * 240.0, 0 if conv == O.CONV_NATIVE else lib.FLAG_SATURATED))
    rows.append((base * 448.0, 0))
    for x, flag in rows:
        case = R.make_case(5, [1], [1], 1, D, 16, conv)
        dev, cache, batch = on_gpu(lib, case, conv, 1, 1)
        k = x.float().cuda().view(1, 1, D)
        v = base.flip(0).float().cuda().view(1, 1, D)
        ctx.device_flags()
        ctx.kv_append(cache, batch, k, v)
        compare_cache(dev, expected_append(case, k.double().cpu().numpy(), v.double().cpu().numpy(), conv))
        got = ctx.device_flags()
        assert got & (lib.FLAG_ZERO_AMAX | lib.FLAG_NONFINITE_AMAX) == flag & (lib.FLAG_ZERO_AMAX | lib.FLAG_NONFINITE_AMAX)
        if flag & lib.FLAG_SATURATED:
            assert got & lib.FLAG_SATURATED


@pytest.mark.parametrize("dim,heads,page,conv", [(64, 3, 16, O.CONV_PAPER), (128, 2, 64, O.CONV_NATIVE), (128, 8, 32, O.CONV_PAPER)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_read_gives_every_number(lib, ctx, dim, heads, page, conv, dtype):
    lens, news = [70, 1, 0, 33, 3], [70, 1, 0, 20, 6]
    case = R.make_case(12, lens, news, heads, dim, page, conv)
    case["bk"][0, 0, :4] = torch.tensor([-128, -121, 64, -30], dtype=torch.int8)
    T = sum(news)
    dev, cache, batch = on_gpu(lib, case, conv, 70, 70)
    out = torch.full((T, 2 * heads + 1, dim), float("nan"), dtype=DT[dtype], device="cuda")
    k, v = out[:, :heads], out[:, heads:2 * heads]
    ctx.kv_read(cache, batch, k, v)
    qs = case["q_start"].numpy()
    cpu = [case[n].numpy() for n in ("k8", "v8", "bk", "bv")]
    for b in range(len(lens)):
        n = news[b]
        pos = np.arange(lens[b] - n, lens[b])
        keep = pos >= 0
        kc, kb, vc, vb = R.cached_rows(cpu, case["table"].numpy(), b, pos[keep])
        for got, codes, bias in ((k, kc, kb), (v, vc, vb)):
            want = np.zeros((n, heads, dim))
            want[keep] = R.numbers(codes, bias, conv)
            w = torch.from_numpy(want).to(torch.float32).to(DT[dtype])
            assert torch.equal(got[qs[b]:qs[b + 1]].cpu(), w)
    assert torch.isnan(out[:, 2 * heads:]).all()
    only = torch.empty((T, heads, dim), dtype=DT[dtype], device="cuda")
    ctx.kv_read(cache, batch, None, only)
    assert torch.equal(only, v.contiguous())


def test_read_after_append_is_within_half_a_step(lib, ctx):
    conv = O.CONV_PAPER
    lens = news = [200, 63]
    case = R.make_case(13, lens, news, 4, 128, 32, conv)
    dev, cache, batch = on_gpu(lib, case, conv, 200, 200)
    k, v = (torch.randn((263, 4, 128), generator=case["g"]).cuda() for _ in range(2))
    ctx.kv_append(cache, batch, k, v)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    ctx.kv_read(cache, batch, k2, v2)
    for x, y in ((k, k2), (v, v2)):
        amax = x.abs().amax(-1, keepdim=True)
        # half a step of three mantissa bits, of the format's subnormals (2^-9 where the amax lies above 120), and the
        # largest numbers lose up to 240 - 224 of 240 (no native code for the paper's 240)
        assert ((x - y).abs() <= torch.maximum(x.abs() / 16, amax * 2.0 ** -15) + (x.abs() > amax * 0.93) * amax / 15).all()


def test_pages_far_apart_and_beyond_32_bits(lib, ctx):
    """A cache of 4.6 GB whose keys and values of a page share one buffer; the tokens lie in its last pages."""
    pages, heads, size, dim, conv = 70000, 2, 128, 128, O.CONV_NATIVE
    both = torch.zeros((pages, 2, heads, size, dim), dtype=torch.uint8, device="cuda")
    biases = torch.zeros((pages, 2, heads, size), dtype=torch.int8, device="cuda")
    assert both.numel() > 1 << 32
    cache = lib.KvCache(both[:, 0], both[:, 1], biases[:, 0], biases[:, 1], conv=conv)
    table = torch.tensor([[pages - 1, pages - 2, 0]], dtype=torch.int32, device="cuda")
    n = 2 * size + 3
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = lib.SeqBatch(torch.tensor([0, n], **i32), torch.tensor([n], **i32), table, max_q_len=n, max_kv_len=n)
    g = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randn((n, heads, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    ctx.kv_append(cache, batch, k, v)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    ctx.kv_read(cache, batch, k2, v2)
    assert ((k - k2).abs() <= k.abs() / 16 + 2.0 ** -9).all() and ((v - v2).abs() <= v.abs() / 16 + 2.0 ** -9).all()
    codes, stored = R.quantise_row(k[size + 5, 1].double().cpu().numpy(), conv)
    assert np.array_equal(both[pages - 2, 0, 1, 5].cpu().numpy(), codes) and int(biases[pages - 2, 0, 1, 5]) == stored
    assert int(both[1:pages - 2].view(-1)[::4097].count_nonzero()) == 0


def test_pages_and_lengths_out_of_bounds_are_flagged(lib, ctx):
    conv = O.CONV_PAPER
    case = R.make_case(14, [40, 40], [40, 40], 2, 64, 16, conv)
    case["table"][0, 1] = 10 ** 6
    case["table"][1, 2] = -5
    dev, cache, batch = on_gpu(lib, case, conv, 40, 40)
    k, v = (torch.randn((80, 2, 64), generator=case["g"]).cuda() for _ in range(2))
    ctx.device_flags()
    ctx.kv_append(cache, batch, k, v)
    want = {n: case[n].numpy().copy() for n in ("k8", "v8", "bk", "bv")}
    for b, i in [(b, i) for b in range(2) for i in range(40) if (b, i // 16) not in ((0, 1), (1, 2))]:
        pg, off = int(case["table"][b, i // 16]), i % 16
        for x, codes, bias in ((k, "k8", "bk"), (v, "v8", "bv")):
            for h in range(2):
                want[codes][pg, h, off], want[bias][pg, h, off] = R.quantise_row(x[40 * b + i, h].double().cpu().numpy(), conv)
    compare_cache(dev, want)
    assert ctx.device_flags() & lib.FLAG_BAD_INDEX
    ctx.kv_read(cache, batch, k, v)
    assert ctx.device_flags() & lib.FLAG_BAD_INDEX
    assert int(k[16:32].count_nonzero()) == 0 and int(v[72:].count_nonzero()) == 0 and int(k[:16].count_nonzero()) > 0
    # a length beyond its bound: the tokens behind it are left out
    case = R.make_case(15, [40], [40], 1, 64, 16, conv)
    dev, cache, batch = on_gpu(lib, case, conv, 40, 33)
    before = dev["k8"].clone()
    ctx.kv_append(cache, batch, k[:40, :1].contiguous(), v[:40, :1].contiguous())
    assert ctx.device_flags() & lib.FLAG_BAD_INDEX
    last = int(case["table"][0, 2])
    assert torch.equal(dev["k8"][last, :, 1:], before[last, :, 1:])


def test_many_sequences_find_their_rows(lib, ctx):
    """More sequences than one round of probes covers, empty ones among them."""
    conv, rng = O.CONV_NATIVE, np.random.default_rng(4)
    news = [int(x) for x in rng.integers(0, 3, 2100)]
    lens = [n + int(e) for n, e in zip(news, rng.integers(0, 4, 2100))]
    case = R.make_case(16, lens, news, 1, 64, 16, conv)
    dev, cache, batch = on_gpu(lib, case, conv, 2, 6)
    T = sum(news)
    k, v = (torch.randn((T, 1, 64), generator=case["g"]).cuda() for _ in range(2))
    ctx.kv_append(cache, batch, k, v)
    compare_cache(dev, expected_append(case, k.double().cpu().numpy(), v.double().cpu().numpy(), conv))


def test_refusals(lib, ctx):
    conv = O.CONV_PAPER
    case = R.make_case(17, [20], [4], 2, 64, 16, conv)
    dev, cache, batch = on_gpu(lib, case, conv, 4, 20)
    k = torch.zeros((4, 2, 64), device="cuda")

    def status(change=None, k=k, **fields):
        c, b = type(cache._desc)(), type(batch._desc)()
        for n, _ in c._fields_:
            setattr(c, n, getattr(cache._desc, n))
        for n, _ in b._fields_:
            setattr(b, n, getattr(batch._desc, n))
        b.tokens = 4
        a = dict(dt=lib.F32, ld=128, conv=conv, kp=k.data_ptr(), vp=k.data_ptr(), ctx=ctx._h)
        for n, x in fields.items():
            if n in a:
                a[n] = x
            else:
                setattr(c if hasattr(c, n) else b, n, x)
        got = []
        for fn in (lib.raw().fp8_kv_append, lib.raw().fp8_kv_read):
            got.append(fn(a["ctx"], c, b, a["kp"], a["vp"], a["dt"], a["ld"], a["ld"], a["conv"], None))
        assert len(set(got)) == 1 or (a["kp"] is None) != (a["vp"] is None)
        return got[0]

    assert status() == lib.OK
    for n in ("k8", "v8", "bk", "bv", "d_q_start", "d_kv_len", "d_page_table", "kp", "ctx"):
        assert status(**{n: None}) == lib.ERR_NULL, n
    for n in ("pages", "kv_heads", "page_size", "head_dim", "seqs", "tokens", "max_q_len", "max_kv_len"):
        assert status(**{n: 0}) == lib.ERR_SHAPE and status(**{n: -3}) == lib.ERR_SHAPE, n
    assert status(head_dim=96) == lib.ERR_UNSUPPORTED and status(page_size=8) == lib.ERR_UNSUPPORTED
    assert status(page_size=48) == lib.ERR_UNSUPPORTED
    assert status(page_stride=2 * 16 * 64 - 16) == lib.ERR_SHAPE and status(bias_stride=16) == lib.ERR_SHAPE
    assert status(table_stride=1) == lib.ERR_SHAPE and status(pages=1 << 28) == lib.ERR_SHAPE
    assert status(page_stride=2 * 16 * 64 + 8) == lib.ERR_ALIGN and status(bias_stride=40) == lib.ERR_ALIGN
    assert status(k8=cache._desc.k8 + 8) == lib.ERR_ALIGN and status(bv=cache._desc.bv + 4) == lib.ERR_ALIGN
    assert status(ld=127) == lib.ERR_SHAPE and status(ld=129) == lib.ERR_ALIGN and status(vp=k.data_ptr() + 4) == lib.ERR_ALIGN
    assert status(dt=3) == lib.ERR_DTYPE and status(conv=2) == lib.ERR_DTYPE
    with pytest.raises(ValueError):
        ctx.kv_append(cache, batch, k.transpose(0, 1), k)
    with pytest.raises(ValueError):
        ctx.kv_append(cache, batch, k, k.bfloat16())
    with pytest.raises(ValueError):
        lib.KvCache(dev["k8"], dev["v8"][:1], dev["bk"], dev["bv"])
    with pytest.raises(ValueError):
        lib.SeqBatch(dev["q_start"].long(), dev["kv_len"], dev["table"], 4, 20)
