"""fp8_norm_fwd and fp8_norm_bwd where their numbers or sizes end.  Tolerances as in test_gpu_norm."""
import pytest
import torch

import head_reference as R
from test_gpu_norm import BF16, F16, F32, U, check_grad, check_norm, inputs, new

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin


@pytest.fixture(scope="module")
def ctx(L):
    return L.Context(0)


# rows of whole vectors (few: one cluster where bytes are wanted; many) by a warp and by several, element by element, walked
ROWS = [(6, 512, BF16), (900, 512, F16), (6, 4096, F32), (300, 5120, BF16), (6, 1027, BF16), (6, 5000, F32), (6, 17000, F16)]


@pytest.mark.parametrize("rows,cols,dtype", ROWS)
@pytest.mark.parametrize("layer", [True, False])
def test_rows_that_are_no_numbers(L, ctx, rows, cols, dtype, layer):
    """A NaN makes its row NaN, the statistics too; so does an infinity in a layer norm.  The root-mean-square form has
    1 / infinity = 0 there: zeros, and NaN in the infinity's place.  Bytes are those of the cast, the other rows as without them."""
    x, res, w, b = inputs(rows, cols, dtype, dtype, cols, True)
    kind, b = (L.NORM_LAYER, b) if layer else (L.NORM_RMS, None)
    good = new(rows, cols, dtype=dtype)
    ctx.norm_fwd(x, w, b, residual=res, kind=kind, y=good)
    x[1, cols // 2], x[2, cols - 1], x[4, 0] = NAN, INF, -INF
    bias = torch.zeros(1, dtype=torch.int32, device="cuda")
    for given in (False, True):
        y, y8, mean, rstd = new(rows, cols, dtype=dtype), new(rows, cols, dtype=torch.uint8), new(rows), new(rows)
        ctx.norm_fwd(x, w, b, residual=res, kind=kind, y=y, d_mean=mean, d_rstd=rstd, y8=y8, d_bias=bias if given else None,
                     d_bias_out=None if given else bias)
        assert given or bias.tolist() == [0]
        bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
        bad[[1, 2, 4]] = True
        assert torch.equal(y[~bad], good[~bad]) and bool((torch.isfinite(rstd[~bad]) & torch.isfinite(mean[~bad])).all())
        if layer:
            assert bool((torch.isnan(y[bad]).all() & torch.isnan(mean[bad]).all() & torch.isnan(rstd[bad]).all()))
        else:
            assert bool(torch.isnan(y[1]).all() and torch.isnan(rstd[1])) and rstd[[2, 4]].tolist() == [0.0, 0.0]
            want = torch.zeros((2, cols), dtype=dtype, device="cuda")
            want[0, cols - 1] = want[1, 0] = NAN
            assert torch.equal(torch.isnan(y[[2, 4]]), torch.isnan(want)) and bool((torch.nan_to_num(y[[2, 4]]) == 0).all())
        want = new(rows, cols, dtype=torch.uint8)
        ctx.cast_e4(y, bias, y=want)
        assert torch.equal(y8, want)
    ctx.device_flags()


@pytest.mark.parametrize("rows,cols,dtype", [(r, c, BF16 if d == F16 else d) for r, c, d in ROWS])
@pytest.mark.parametrize("layer", [True, False])
def test_rows_whose_squares_fp32_does_not_hold(L, ctx, rows, cols, dtype, layer):
    """Without eps a norm does not know its input's scale: a row times 2^k gives the same bits, its statistics times 2^k and
    2^-k, whether the squares pass FP32 (k = 70, 110), are subnormal (-75) or nothing (-100).  Rows of ordinary size beside them
    are what they were, and with an eps the definition holds."""
    x, res, w, b = inputs(rows, cols, dtype, dtype, 2 * cols, True)
    x, res = (torch.where(t.abs() < 2.0 ** -10, torch.ones_like(t), t) for t in (x, res))   # (nothing becomes subnormal)
    kind, b = (L.NORM_LAYER, b) if layer else (L.NORM_RMS, None)

    def run(x, res, eps):
        out = dict(h=new(rows, cols, dtype=dtype), y=new(rows, cols, dtype=dtype), d_mean=new(rows), d_rstd=new(rows),
                   y8=new(rows, cols, dtype=torch.uint8), d_bias_out=new(1, dtype=torch.int32))
        ctx.norm_fwd(x, w, b, residual=res, kind=kind, eps=eps, **out)
        return out
    want = run(x, res, 0.0)
    check_norm(*R.norm(x, w, b, res, eps=0.0, layer=layer), w, b, layer, dtype, want["h"], want["y"], want["d_mean"], want["d_rstd"])
    for k in (70, 110, -75, -100):
        by = torch.ones((rows, 1), device="cuda")
        by[1::2] = 2.0 ** k
        got = run((x.float() * by).to(dtype), (res.float() * by).to(dtype), 0.0)
        assert torch.equal(got["h"].float(), want["h"].float() * by)
        assert torch.equal(got["d_mean"], want["d_mean"] * by[:, 0]) and torch.equal(got["d_rstd"] * by[:, 0], want["d_rstd"])
        assert all(torch.equal(got[n], want[n]) for n in ("y", "y8", "d_bias_out")), k
        place, y = (x.float() * by).to(dtype), new(rows, cols, dtype=dtype)   # (the sum in x's place, and only y beside it)
        ctx.norm_fwd(place, w, b, residual=(res.float() * by).to(dtype), kind=kind, eps=0.0, h=place, y=y)
        assert torch.equal(place, got["h"]) and torch.equal(y, want["y"])
    large = (x.float() * 2.0 ** 100).to(dtype)
    got = run(large, None, 1e-5)
    check_norm(*R.norm(large, w, b, layer=layer), w, b, layer, dtype, None, got["y"], got["d_mean"], got["d_rstd"])


def test_sums_that_fp32_does_not_hold(L, ctx):
    """Rows whose plain sum passes FP32, up to the type's largest number."""
    for cols in (512, 4096, 1027):
        x = torch.linspace(0.5, 1.0, cols, device="cuda").repeat(3, 1)
        x[1] *= torch.finfo(BF16).max
        x[2] = torch.finfo(BF16).max
        x = x.to(BF16)
        y, mean, rstd = new(3, cols, dtype=BF16), new(3), new(3)
        ctx.norm_fwd(x, y=y, d_mean=mean, d_rstd=rstd)
        assert bool(torch.isinf(x[1:].float().sum(-1)).all())
        check_norm(*R.norm(x), None, None, True, BF16, None, y, mean, rstd)
        assert bool((y[2] == 0).all()) and float(mean[2]) == torch.finfo(BF16).max


@pytest.mark.parametrize("rows,cols", [(1, (1 << 23) + 8), (3, (1 << 24) + 1), (2, 1 << 22)])
@pytest.mark.parametrize("layer", [True, False])
def test_gradient_of_very_long_rows(L, ctx, rows, cols, layer):
    """Without dw and db no workspace is asked for, and rows are as long as they like."""
    h, dy, _, _ = inputs(rows, cols, BF16, BF16, 21, True)
    _, _, mean, rstd = R.norm(h, layer=layer)
    dx = new(rows, cols, dtype=BF16)
    ctx.norm_bwd(dy, h, None, mean.float() if layer else None, rstd.float(), dx, kind=L.NORM_LAYER if layer else L.NORM_RMS)
    check_grad(dx, R.norm_grad(dy, h, None, layer=layer)[0], None, dy, h, None, rstd, BF16)


@pytest.mark.parametrize("cols,dtype", [(512, BF16), (4096, F16), (14272, F32), (16384, F32), (16384, BF16)])
def test_a_row_has_the_same_bits_in_every_call(L, ctx, cols, dtype):
    """Aligned rows with a residual: statistics and output do not depend on how many rows the call has, nor on whether bytes are
    asked for beside it."""
    x, res, w, b = inputs(40, cols, dtype, dtype, 22, True)
    y, mean, rstd = new(40, cols, dtype=dtype), new(40), new(40)
    ctx.norm_fwd(x, w, b, residual=res, y=y, d_mean=mean, d_rstd=rstd)
    for n in (1, 2, 8, 40):
        got, m, s, y8, bias = new(n, cols, dtype=dtype), new(n), new(n), new(n, cols, dtype=torch.uint8), new(1, dtype=torch.int32)
        ctx.norm_fwd(x[:n], w, b, residual=res[:n], d_mean=m, d_rstd=s, y8=y8, d_bias_out=bias)
        want = new(n, cols, dtype=torch.uint8)
        ctx.cast_e4(y[:n], bias, y=want)
        assert torch.equal(m, mean[:n]) and torch.equal(s, rstd[:n]) and torch.equal(y8, want), n
        ctx.norm_fwd(x[:n], w, b, residual=res[:n], y=got)
        assert torch.equal(got, y[:n]), n
    ctx.device_flags()


@pytest.mark.parametrize("rows,cols,dtype", [(300, 512, BF16), (700, 4096, F32), (300, 8192, F16), (40, 16384, F32), (60, 1027, BF16)])
def test_row_sums_with_and_without_a_joining_gradient(L, ctx, rows, cols, dtype):
    """dw and db do not contain dh.  (Which rows are summed together may depend on it: FP32 rows leave room for fewer groups.)"""
    h, dy, w, _ = inputs(rows, cols, dtype, dtype, 23, True)
    dh = inputs(rows, cols, dtype, dtype, 24, False)[0]
    _, _, mean, rstd = (t.float() for t in R.norm(h))
    _, want_w, want_b = R.norm_grad(dy, h, w)
    xh = ((h.double() - mean.double().unsqueeze(-1)).abs() + h.double().abs()) * rstd.double().unsqueeze(-1)
    for join in (None, dh):
        dx, dw, db = new(rows, cols, dtype=dtype), new(cols, dtype=dtype), new(cols, dtype=dtype)
        ctx.norm_bwd(dy, h, w, mean, rstd, dx, dh=join, dw=dw, db=db)
        check_grad(dx, R.norm_grad(dy, h, w, join)[0], join, dy, h, w, rstd, dtype)
        for got, ref, size in ((dw, want_w, (dy.double().abs() * xh).sum(0)), (db, want_b, dy.double().abs().sum(0))):
            d = size * (rows + 40) * U + ref.abs() * R.HALF[dtype] + R.TINY[dtype]
            assert bool(((got.double() - ref).abs() <= d).all())


@pytest.mark.parametrize("rows,cols,dtype", [(r, c, BF16 if d == F16 else d) for r, c, d in ROWS])
def test_large_numbers_of_little_spread(L, ctx, rows, cols, dtype):
    """No spread to speak of is not the same as small numbers: rows of one number, 2^-40 to 2^120, keep their mean and, with any
    eps, give zeros; rows of numbers below 2^-60 with a mean far above their spread."""
    x = torch.exp2(torch.linspace(-40, 120, rows, device="cuda")).unsqueeze(1).expand(rows, cols).to(dtype).contiguous()
    for eps in (1e-30, 1e-5):
        y, mean, rstd = new(rows, cols, dtype=dtype), new(rows), new(rows)
        ctx.norm_fwd(x, eps=eps, y=y, d_mean=mean, d_rstd=rstd, y8=new(rows, cols, dtype=torch.uint8), d_bias_out=new(1, dtype=torch.int32))
        assert bool((y == 0).all()) and torch.equal(mean, x[:, 0].float())
        assert bool(((rstd.double() * eps ** 0.5 - 1).abs() <= 4 * U).all())
    ctx.norm_fwd(x, eps=0.0, d_mean=mean)
    assert torch.equal(mean, x[:, 0].float())
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = ((1 + torch.randn((rows, cols), generator=g, device="cuda") / 32) * 2.0 ** -70).to(dtype)
    ctx.norm_fwd(x, eps=0.0, y=y, d_mean=mean, d_rstd=rstd)
    # (the mean's own rounding, 32 spreads of it, is what `path` allows relative to the size)
    check_norm(*R.norm(x, eps=0.0), None, None, True, dtype, None, y, mean, rstd)
    ctx.device_flags()
