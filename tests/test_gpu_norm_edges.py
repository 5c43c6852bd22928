"""fp8_norm_fwd and fp8_norm_bwd where their numbers or sizes end.  Tolerances as in test_gpu_norm."""
import pytest
import torch

import head_reference as R
from test_gpu_norm import BF16, F16, F32, inputs, new

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
