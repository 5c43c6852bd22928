"""fp8_norm_fwd and fp8_norm_bwd against the definitions in 64 bits.

Tolerances count roundings of 2^-24 (FP32) and one of the output's type.  A sum of n terms adds at most n/256 + 32 of them on
one path: a thread adds its terms (32 as two sums of 16: 17), a warp joins its lanes in 5, a block its warps one after the other.
Whole vectors: a warp alone 22 (up to 1024 terms), 128 threads 25 (4096), 256 threads 29, 512 threads 37 (from 8193 on: 64 allowed).
Element by element: 64 threads 14, 256 threads 20, 512 threads 28, 1024 threads 44 (from 4097 on: 48 allowed) or 52 (from 8193
on); walked rows n/256 + 5 + 7."""
import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def L():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin


@pytest.fixture(scope="module")
def ctx(L):
    return L.Context(0)


def new(*shape, dtype=F32):
    t = torch.empty(shape, dtype=dtype, device="cuda")
    return t.view(torch.uint8).fill_(0xA5).view(dtype).view(shape) if t.numel() else t


def inputs(rows, cols, dtype, w_dtype, seed, residual, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    def one(offset):
        t = torch.randn((rows, ld or cols), generator=g, device="cuda") * 2 + offset
        t[:, ::7] *= 20
        return t.to(dtype)[:, :cols]
    x, res = one(0.5), one(-0.3) if residual else None
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(w_dtype)
    b = (0.2 * torch.randn(cols, generator=g, device="cuda")).to(w_dtype)
    return x, res, w, b


def path(cols):
    """Roundings on the longest path of a sum over a row."""
    return cols / 256 + 32


def check_norm(h, y, mean, rstd, w, b, layer, dtype, got_h, got_y, got_mean, got_rstd):
    if got_h is not None:
        assert torch.equal(got_h, h)
    cols, h64 = h.shape[1], h.double()
    size = h64.abs().mean(-1)                                    # a sum's error is relative to the sum of magnitudes
    d_mean = (path(cols) + 2) * U * size if layer else torch.zeros_like(size)
    # variance: its own sum, and the mean's error squared is far below; rsqrt: half of that, division and root two more
    d_rstd = (path(cols) / 2 + 6) * U * rstd + rstd * (d_mean * rstd) ** 2
    if layer:
        assert bool(((got_mean.double() - mean).abs() <= d_mean).all())
    assert bool(((got_rstd.double() - rstd).abs() <= d_rstd).all())
    if got_y is None:
        return
    xh = (h64 - mean.unsqueeze(-1)) * rstd.unsqueeze(-1)
    w = torch.ones(cols, dtype=torch.float64, device="cuda") if w is None else w.double()
    d = ((d_mean * rstd).unsqueeze(-1) + xh.abs() * ((d_rstd / rstd).unsqueeze(-1) + 3 * U) + (h64.abs() * rstd.unsqueeze(-1)) * U) * w.abs()
    d = d + y.abs() * (R.HALF[dtype] + U) + R.TINY[dtype]
    assert bool(((got_y.double() - y).abs() <= d).all()), float(((got_y.double() - y).abs() / d).max())


SIZES = [(1, 1), (3, 2), (5, 7), (1, 64), (4, 512), (9, 520), (2, 1000), (3, 1027), (300, 1024), (7, 4096), (1201, 4096), (33, 5120),
         (17, 8192), (6, 11008), (5, 16384), (3, 16392), (2, 40000)]


@pytest.mark.parametrize("dtype,w_dtype", [(BF16, BF16), (F16, F16), (F32, F32), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(L, ctx, rows, cols, layer, dtype, w_dtype):
    for residual, ld in ((True, None), (False, cols + 24), (True, cols + 3)):
        x, res, w, b = inputs(rows, cols, dtype, w_dtype, rows + cols, residual, ld)
        if not layer:
            b = None
        h, y, mean, rstd = new(rows, cols, dtype=dtype), new(rows, cols, dtype=dtype), new(rows), new(rows)
        ctx.norm_fwd(x, w, b, residual=res, kind=L.NORM_LAYER if layer else L.NORM_RMS, h=h if residual else None, y=y, d_mean=mean,
                     d_rstd=rstd)
        check_norm(*R.norm(x, w, b, res, layer=layer), w, b, layer, dtype, h if residual else None, y, mean, rstd)
        if not layer:
            assert bool((mean == 0).all())


@pytest.mark.parametrize("conv", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 64), (1, 8192), (4, 512), (16, 8192), (64, 4096), (129, 1024), (7, 1027), (700, 4096), (2500, 2048)])
def test_bytes_are_those_of_the_cast(L, ctx, rows, cols, dtype, conv):
    """Bytes, amax and bias, bit for bit those that fp8_cast_e4 makes of the call's own y; with and without y, residual and
    a stored sum."""
    x, res, w, b = inputs(rows, cols, dtype, dtype, 3 * rows + cols, True)
    for kind, margin in ((L.NORM_LAYER, 0), (L.NORM_RMS, 2)):
        vec = b if kind == L.NORM_LAYER else None
        y, y8, mean, rstd = new(rows, cols, dtype=dtype), new(rows, cols, dtype=torch.uint8), new(rows), new(rows)
        h, amax, bias = new(rows, cols, dtype=dtype), new(1), new(1, dtype=torch.int32)
        ctx.norm_fwd(x, w, vec, residual=res, kind=kind, h=h, y=y, d_mean=mean, d_rstd=rstd, y8=y8, d_amax_out=amax, d_bias_out=bias,
                     conv=conv, margin=margin)
        want, want_amax, want_bias = new(rows, cols, dtype=torch.uint8), new(1), new(1, dtype=torch.int32)
        ctx.cast_e4(y, None, conv=conv, margin=margin, d_amax_out=want_amax, d_bias_out=want_bias, y=want)
        assert torch.equal(amax, want_amax) and torch.equal(bias, want_bias) and torch.equal(y8, want)
        check_norm(*R.norm(x, w, vec, res, layer=kind == L.NORM_LAYER), w, vec, kind == L.NORM_LAYER, dtype, h, y, mean, rstd)
        # nothing but the bytes is kept, the sum neither
        again, amax2, bias2 = new(rows, cols, dtype=torch.uint8), new(1), new(1, dtype=torch.int32)
        ctx.norm_fwd(x, w, vec, residual=res, kind=kind, d_mean=mean, d_rstd=rstd, y8=again, d_amax_out=amax2, d_bias_out=bias2, conv=conv,
                     margin=margin)
        assert torch.equal(again, want) and torch.equal(amax2, want_amax) and torch.equal(bias2, want_bias)
        # a given bias: one pass, the amax beside it, bias_out of that amax
        given = want_bias + 3
        ctx.cast_e4(y, given, conv=conv, y=want)
        ctx.norm_fwd(x, w, vec, residual=res, kind=kind, y8=again, d_bias=given, d_amax_out=amax2, d_bias_out=bias2, conv=conv, margin=margin)
        assert torch.equal(again, want) and torch.equal(amax2, want_amax) and torch.equal(bias2, want_bias)
    ctx.device_flags()


def test_flags_follow_the_cast(L, ctx):
    x = torch.zeros((3, 64), dtype=BF16, device="cuda")
    y8, mean, rstd, bias = new(3, 64, dtype=torch.uint8), new(3), new(3), new(1, dtype=torch.int32)
    ctx.device_flags()
    ctx.norm_fwd(x, d_mean=mean, d_rstd=rstd, y8=y8, d_bias_out=bias)
    assert ctx.device_flags() == L.FLAG_ZERO_AMAX and bias.tolist() == [0] and bool((y8 == 0).all())
    x[1, 5] = float("inf")
    ctx.norm_fwd(x, d_mean=mean, d_rstd=rstd, y8=y8, d_bias_out=bias)
    assert ctx.device_flags() & L.FLAG_NONFINITE_AMAX and bias.tolist() == [0]
    x = torch.randn((3, 64), device="cuda").to(BF16)
    ctx.norm_fwd(x, y8=y8, d_bias=torch.tensor([12], dtype=torch.int32, device="cuda"))
    assert ctx.device_flags() == L.FLAG_SATURATED


def test_a_bad_row_stays_alone(L, ctx):
    x, res, w, b = inputs(20, 1024, BF16, BF16, 5, True)
    good, y = new(20, 1024, dtype=BF16), new(20, 1024, dtype=BF16)
    ctx.norm_fwd(x, w, b, residual=res, y=good)
    x[3, 7], x[9, 1023], x[15, 0] = float("nan"), float("inf"), float("-inf")
    ctx.norm_fwd(x, w, b, residual=res, y=y)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[[3, 9, 15]] = True
    assert torch.equal(y[~bad], good[~bad]) and bool(torch.isnan(y[bad]).all())


def test_large_numbers_and_none(L, ctx):
    """Constant rows, rows of zeros, a mean far above the spread (deviations are taken from the mean, not from zero)."""
    x = torch.full((4, 512), 1000.0, device="cuda")
    x[0] = 0.0
    x[2] += torch.linspace(-1, 1, 512, device="cuda")
    x[3] = 1e15
    y, mean, rstd = new(4, 512), new(4), new(4)
    ctx.norm_fwd(x, y=y, d_mean=mean, d_rstd=rstd)
    assert bool((y[[0, 1, 3]] == 0).all()) and mean.tolist()[:2] == [0.0, 1000.0]
    check_norm(*R.norm(x[2:3]), None, None, True, F32, None, y[2:3], mean[2:3], rstd[2:3])


def test_the_sum_may_take_an_input_s_place(L, ctx):
    for cols in (1024, 1027):
        x, res, w, b = inputs(9, cols, BF16, BF16, 6, True)
        want, y1, y2 = new(9, cols, dtype=BF16), new(9, cols, dtype=BF16), new(9, cols, dtype=BF16)
        ctx.norm_fwd(x, w, b, residual=res, h=want, y=y1)
        for place in (0, 1):
            a, r = x.clone(), res.clone()
            ctx.norm_fwd(a, w, b, residual=r, h=(a, r)[place], y=y2)
            assert torch.equal((a, r)[place], want) and torch.equal(y2, y1) and torch.equal((r, a)[place], (res, x)[place])


BWD = [(1, 1), (2, 3), (4, 64), (9, 520), (130, 512), (3, 1027), (900, 1024), (257, 2048), (1201, 4096), (20, 5120), (40, 8192), (6, 11008),
       (5, 16384), (3, 16392), (2, 40000)]


def check_grad(got, want, dh, dy, h, w, rstd, dtype):
    """dx = rstd (g - c1 - xh c2): c1 and c2 carry a sum's error, the statistics theirs."""
    cols = h.shape[1]
    g = (dy.double() if w is None else dy.double() * w.double()).abs()
    xh = (h.double() - h.double().mean(-1, keepdim=True)).abs() * rstd.double().unsqueeze(-1) + h.double().abs() * rstd.double().unsqueeze(-1)
    one = g.mean(-1, keepdim=True) + xh * (g * xh).mean(-1, keepdim=True) + g
    d = rstd.double().unsqueeze(-1) * one * (2 * path(cols) + 16) * U + (want.abs() + (0 if dh is None else dh.double().abs())) * 2 * U
    d = d + want.abs() * R.HALF[dtype] + R.TINY[dtype]
    assert bool(((got.double() - want).abs() <= d).all()), float(((got.double() - want).abs() / d).max())


@pytest.mark.parametrize("dtype,w_dtype", [(BF16, BF16), (F16, F16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("rows,cols", BWD)
def test_backward(L, ctx, rows, cols, layer, dtype, w_dtype):
    kind = L.NORM_LAYER if layer else L.NORM_RMS
    for join, ld in ((True, None), (False, cols + 24), (True, cols + 5)):
        h, dy, w, _ = inputs(rows, cols, dtype, w_dtype, rows * 3 + cols, True, ld)
        dh = inputs(rows, cols, dtype, w_dtype, rows * 5 + cols, False, ld)[0] if join else None
        _, _, mean, rstd = R.norm(h, layer=layer)
        mean, rstd = mean.float(), rstd.float()
        dx, dw, db, amax = new(rows, cols, dtype=dtype), new(cols, dtype=w_dtype), new(cols, dtype=w_dtype), new(1)
        ctx.norm_bwd(dy, h, w, mean if layer else None, rstd, dx, dh=dh, dw=dw, db=db, d_amax=amax, kind=kind)
        want, want_w, want_b = R.norm_grad(dy, h, w, dh, layer=layer)
        check_grad(dx, want, dh, dy, h, w, rstd, dtype)
        assert float(amax) == float(dx.float().abs().max())
        # sums over rows: at most rows + 8 + the joins of the parts on one path; xh carries 4 roundings and its statistics' 2
        xh = (h.double() - (mean.double().unsqueeze(-1) if layer else 0)).abs() * rstd.double().unsqueeze(-1) + h.double().abs() * rstd.double().unsqueeze(-1)
        for got, ref, size in ((dw, want_w, (dy.double().abs() * xh).sum(0)), (db, want_b, dy.double().abs().sum(0))):
            d = size * (rows + 40) * U + ref.abs() * R.HALF[w_dtype] + R.TINY[w_dtype]
            assert bool(((got.double() - ref).abs() <= d).all()), float(((got.double() - ref).abs() / d).max())


def test_backward_parts(L, ctx):
    """Any of the three outputs alone gives the same bits; no weight counts as ones; dx may take dy's or dh's place."""
    for cols in (1024, 1027, 5120):
        h, dy, w, _ = inputs(70, cols, BF16, BF16, 8, True)
        dh = inputs(70, cols, BF16, BF16, 9, False)[0]
        _, _, mean, rstd = (t.float() for t in R.norm(h))
        dx, dw, db = new(70, cols, dtype=BF16), new(cols, dtype=BF16), new(cols, dtype=BF16)
        ctx.norm_bwd(dy, h, w, mean, rstd, dx, dh=dh, dw=dw, db=db)
        for part in range(3):
            out = [new(70, cols, dtype=BF16), new(cols, dtype=BF16), new(cols, dtype=BF16)]
            ctx.norm_bwd(dy, h, w, mean, rstd, out[0] if part == 0 else None, dh=dh, dw=out[1] if part == 1 else None,
                         db=out[2] if part == 2 else None)
            assert torch.equal(out[part], (dx, dw, db)[part])
        for place in (0, 1):
            a, b = dy.clone(), dh.clone()
            ctx.norm_bwd(a, h, w, mean, rstd, (a, b)[place], dh=b)
            assert torch.equal((a, b)[place], dx)
        plain, ones = new(70, cols, dtype=BF16), new(70, cols, dtype=BF16)
        ctx.norm_bwd(dy, h, None, mean, rstd, plain)
        ctx.norm_bwd(dy, h, torch.ones(cols, device="cuda"), mean, rstd, ones)
        assert torch.equal(plain, ones)


def test_gradient_is_the_slope_of_the_forward_call(L, ctx):
    """Differences of the forward call itself, FP32: step 2^-6, error of third derivatives about 2^-12 of the value, rounding
    2^-24 * sqrt(cols) / 2^-6 of it."""
    g = torch.Generator(device="cuda").manual_seed(10)
    h, dy, u = (torch.randn((6, 512), generator=g, device="cuda") for _ in range(3))
    w = 1 + 0.3 * torch.randn(512, generator=g, device="cuda")
    for kind in (L.NORM_LAYER, L.NORM_RMS):
        def forward(t):
            y = new(6, 512)
            ctx.norm_fwd(t, w, kind=kind, y=y)
            return (y.double() * dy.double()).sum(-1)
        mean, rstd, y, dx = new(6), new(6), new(6, 512), new(6, 512)
        ctx.norm_fwd(h, w, kind=kind, y=y, d_mean=mean, d_rstd=rstd)
        ctx.norm_bwd(dy, h, w, mean, rstd, dx, kind=kind)
        step = 2.0 ** -6
        slope = (forward(h + step * u) - forward(h - step * u)) / (2 * step)
        want = (dx.double() * u.double()).sum(-1)
        assert float((slope - want).abs().max()) < 2.0 ** -9 * float(dx.double().norm() * u.double().norm()) / 6 ** 0.5


def test_rows_far_apart(L, ctx):
    """Row distances that pass 32 bits."""
    ld = 1 << 29
    base = torch.empty(4 * ld + 64, dtype=BF16, device="cuda")
    x = base.as_strided((5, 64), (ld, 1))
    want, _, w, b = inputs(5, 64, BF16, BF16, 11, False)
    x.copy_(want)
    y, ref, mean, rstd = new(5, 64, dtype=BF16), new(5, 64, dtype=BF16), new(5), new(5)
    ctx.norm_fwd(x, w, b, y=y, d_mean=mean, d_rstd=rstd)
    ctx.norm_fwd(want, w, b, y=ref)
    assert torch.equal(y, ref)
    dx, far = new(5, 64, dtype=BF16), x
    ctx.norm_bwd(want, want, w, mean, rstd, dx)
    ctx.norm_bwd(far, far, w, mean, rstd, far)
    assert torch.equal(far, dx)


def test_equal_bits_from_run_to_run_and_from_a_graph(L, ctx):
    x, res, w, b = inputs(3000, 1024, BF16, BF16, 12, True)
    dy = inputs(3000, 1024, BF16, BF16, 13, False)[0]
    h, y8, mean, rstd = new(3000, 1024, dtype=BF16), new(3000, 1024, dtype=torch.uint8), new(3000), new(3000)
    amax, bias, dx, dw, db = new(1), new(1, dtype=torch.int32), new(3000, 1024, dtype=BF16), new(1024, dtype=BF16), new(1024, dtype=BF16)
    outs = (h, y8, mean, rstd, amax, bias, dx, dw, db)

    def step():
        ctx.norm_fwd(x, w, b, residual=res, h=h, d_mean=mean, d_rstd=rstd, y8=y8, d_amax_out=amax, d_bias_out=bias)
        ctx.norm_bwd(dy, h, w, mean, rstd, dx, dh=x, dw=dw, db=db)
    step()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for run in (step, graph.replay, graph.replay, step, graph.replay):
        for t in outs:
            t.view(torch.uint8).fill_(0x5A)
        run()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, want))


def test_neighbours_stay(L, ctx):
    """Nothing outside the outputs is written (odd and even sizes, rows with a gap)."""
    for rows, cols in ((5, 1027), (5, 1024), (1, 8192), (300, 513)):
        x, res, w, b = inputs(rows, cols, BF16, BF16, 14, True)
        big = {k: new(rows + 2, cols + 16, dtype=d) for k, d in (("h", BF16), ("y", BF16), ("dx", BF16))}
        bytes_ = new((rows + 2) * cols, dtype=torch.uint8)
        vec = {k: new(n + 16, dtype=d) for k, n, d in (("mean", rows, F32), ("rstd", rows, F32), ("dw", cols, BF16), ("db", cols, BF16))}
        before = [t.clone() for t in (*big.values(), bytes_, *vec.values())]
        view = {k: t[1:rows + 1, 8:cols + 8] for k, t in big.items()}
        y8 = bytes_[cols:(rows + 1) * cols].view(rows, cols)
        part = {k: t[8:8 + (rows if k in ("mean", "rstd") else cols)] for k, t in vec.items()}
        ctx.norm_fwd(x, w, b, residual=res, h=view["h"], y=view["y"], d_mean=part["mean"], d_rstd=part["rstd"], y8=y8, d_bias_out=new(1, dtype=torch.int32))
        ctx.norm_bwd(x, view["h"], w, part["mean"], part["rstd"], view["dx"], dw=part["dw"], db=part["db"])
        for t, old in zip((*view.values(), y8, *part.values()), (*[b[1:rows + 1, 8:cols + 8] for b in before[:3]], before[3][cols:(rows + 1) * cols].view(rows, cols),
                                                                *[b[8:8 + len(part[k])] for k, b in zip(part, before[4:])])):
            t.copy_(old)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((*big.values(), bytes_, *vec.values()), before))


def test_many_short_rows_and_long_ones(L, ctx):
    for rows, cols, dtype in ((200001, 8, BF16), (100003, 3, F32), (2, 1 << 20, BF16), (2, (1 << 20) + 1, F16), (3, 16384, F32)):
        x, res, w, b = inputs(rows, cols, dtype, dtype, 15, True)
        h, y, mean, rstd = new(rows, cols, dtype=dtype), new(rows, cols, dtype=dtype), new(rows), new(rows)
        ctx.norm_fwd(x, w, b, residual=res, h=h, y=y, d_mean=mean, d_rstd=rstd)
        check_norm(*R.norm(x, w, b, res), w, b, True, dtype, h, y, mean, rstd)
        dx, dw, db = new(rows, cols, dtype=dtype), new(cols, dtype=dtype), new(cols, dtype=dtype)
        ctx.norm_bwd(x, h, w, mean, rstd, dx, dh=res, dw=dw, db=db)
        want, want_w, want_b = R.norm_grad(x, h, w, res)
        check_grad(dx, want, res, x, h, w, rstd, dtype)
        xh = ((h.double() - mean.double().unsqueeze(-1)).abs() + h.double().abs()) * rstd.double().unsqueeze(-1)
        for got, ref, size in ((dw, want_w, (x.double().abs() * xh).sum(0)), (db, want_b, x.double().abs().sum(0))):
            # (a block's rows one after the other, then 32 sums of the blocks' lines)
            d = size * (rows / 100 + 80) * U + ref.abs() * R.HALF[dtype] + R.TINY[dtype]
            assert bool(((got.double() - ref).abs() <= d).all()), float(((got.double() - ref).abs() / d).max())


def test_forward_calls_on_two_streams_at_once(L, ctx):
    """The forward call has no workspace: two streams may make it on one context at the same time."""
    sets = [inputs(n, 2048, BF16, BF16, 16 + n, True) for n in (600, 9)]

    def run(i):
        x, res, w, b = sets[i]
        n = x.shape[0]
        out = [new(n, 2048, dtype=BF16), new(n, 2048, dtype=torch.uint8), new(n), new(n), new(1), new(1, dtype=torch.int32)]
        ctx.norm_fwd(x, w, b, residual=res, h=out[0], y8=out[1], d_mean=out[2], d_rstd=out[3], d_amax_out=out[4], d_bias_out=out[5])
        return out
    want = run(0), run(1)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [], []
    for _ in range(15):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(run(i))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for r in got[i] for a, b in zip(r, want[i]))
