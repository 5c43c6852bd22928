"""Arguments of the norm and loss calls that are refused: by the binding (tensors that only claim to be on a GPU) and by the
library before it touches a device."""
import ctypes

import pytest
import torch

from paper_2309_17224_b200 import build as B

B.build()
from paper_2309_17224_b200 import fp8lin

BF16, F32 = torch.bfloat16, torch.float32


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def zeros(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def ctx(monkeypatch):
    for name in ("fp8_norm_fwd", "fp8_norm_bwd", "fp8_token_logprobs", "fp8_token_logprobs_bwd", "fp8_distill_fwd", "fp8_distill_bwd"):
        monkeypatch.setattr(fp8lin._lib, name, lambda *a, name=name: pytest.fail(f"{name} was called"))
    c = object.__new__(fp8lin.Context)
    c._h, c.device = None, 0
    return c


X, V, S = zeros(4, 32), zeros(32), zeros(4, dtype=F32)
HOST = torch.zeros((4, 32), dtype=BF16)


@pytest.mark.parametrize("change", [
    dict(x=HOST), dict(x=zeros(32)), dict(x=zeros(4, 32, dtype=torch.float64)), dict(x=zeros(32, 4).t()), dict(residual=zeros(4, 31)),
    dict(residual=zeros(4, 32, dtype=F32)), dict(residual=zeros(1, 32).expand(4, 32)), dict(weight=zeros(31)), dict(weight=zeros(32, dtype=torch.float16)), dict(bias_vec=zeros(32, dtype=F32)),
    dict(weight=zeros(64)[::2]), dict(y=zeros(4, 32, dtype=F32)), dict(h=HOST), dict(d_mean=S[:3]), dict(d_rstd=zeros(4)),
    dict(y8=zeros(4, 32)), dict(y8=zeros(4, 48, dtype=torch.uint8)[:, :32]), dict(d_bias=zeros(1, dtype=F32)), dict(d_amax_out=zeros(2, dtype=F32)),
    dict(d_bias_out=torch.zeros(1, dtype=torch.int32))])
def test_norm_forward(ctx, change):
    args = dict(x=X, weight=V, bias_vec=V, y=X)
    args.update(change)
    with pytest.raises(ValueError):
        ctx.norm_fwd(**args)


@pytest.mark.parametrize("change", [
    dict(dy=HOST), dict(h=zeros(4, 32, dtype=F32)), dict(h=zeros(5, 32)), dict(dh=zeros(4, 31)), dict(weight=zeros(33)), dict(dw=zeros(32, dtype=F32)),
    dict(db=zeros(31)), dict(d_mean=zeros(4)), dict(d_rstd=S[:2]), dict(dx=zeros(4, 32, dtype=torch.float16)), dict(d_amax=zeros(1))])
def test_norm_backward(ctx, change):
    args = dict(dy=X, h=X, weight=V, d_mean=S, d_rstd=S, dx=X, dw=V, db=V)
    args.update(change)
    with pytest.raises(ValueError):
        ctx.norm_bwd(**args)


T, P = zeros(4, dtype=torch.int64), zeros(4, 4, dtype=F32)


@pytest.mark.parametrize("change", [
    dict(logits=HOST), dict(logits=zeros(32)), dict(targets=zeros(4, dtype=torch.int16)), dict(targets=zeros(5, dtype=torch.int64)), dict(logprob=zeros(4)),
    dict(entropy=S[:3]), dict(lse=torch.zeros(4)), dict(saved=zeros(4, 3, dtype=F32)), dict(saved=zeros(4, 8, dtype=F32)[:, :4]),
    dict(top_logprob=zeros(4, 2, dtype=F32)), dict(top_index=zeros(4, 2, dtype=torch.int64)),
    dict(top_logprob=zeros(4, 2, dtype=F32), top_index=zeros(4, 2, dtype=torch.int32)),
    dict(top_logprob=zeros(4, 2, dtype=F32), top_index=zeros(4, 3, dtype=torch.int64))])
def test_token_logprobs(ctx, change):
    args = dict(logits=X, targets=T, logprob=S)
    args.update(change)
    with pytest.raises(ValueError):
        ctx.token_logprobs(**args)


@pytest.mark.parametrize("change", [
    dict(targets=T[:3]), dict(saved=S), dict(dlogits=zeros(4, 33)), dict(dlogits=zeros(4, 32, dtype=F32)), dict(g_logprob=zeros(4)),
    dict(g_entropy=S[:3]), dict(d_amax=S)])
def test_token_logprobs_backward(ctx, change):
    args = dict(logits=X, targets=T, saved=P, dlogits=X, g_logprob=S)
    args.update(change)
    with pytest.raises(ValueError):
        ctx.token_logprobs_bwd(**args)


@pytest.mark.parametrize("change", [
    dict(index=T), dict(index=zeros(3, 2, dtype=torch.int64)), dict(index=zeros(4, 2)), dict(value=zeros(4, 3, dtype=F32)), dict(value=zeros(4, 2)),
    dict(saved=S), dict(logits=zeros(4, 32, dtype=torch.int32))])
def test_distillation(ctx, change):
    args = dict(logits=X, index=zeros(4, 2, dtype=torch.int64), value=zeros(4, 2, dtype=F32))
    args.update(change)
    with pytest.raises(ValueError):
        ctx.distill_fwd(loss=S, **args)
    with pytest.raises(ValueError):
        ctx.distill_bwd(g_loss=S, dlogits=X, **{"saved": P, **args})


def test_calls_without_rows_launch_nothing(ctx):
    x, s, i, v, keep = zeros(0, 32), zeros(0, dtype=F32), zeros(0, 2, dtype=torch.int64), zeros(0, 2, dtype=F32), zeros(0, 4, dtype=F32)
    dw = zeros(32) + 1
    dw = dw.as_subclass(OnGpu)
    ctx.norm_fwd(x, V, V, y=x)
    ctx.norm_bwd(x, x, V, s, s, x, dw=dw)
    assert bool((torch.Tensor(dw.float()) == 0).all())
    ctx.token_logprobs(x, zeros(0, dtype=torch.int64), logprob=s)
    ctx.token_logprobs_bwd(x, zeros(0, dtype=torch.int64), keep, x, g_logprob=s)
    ctx.distill_fwd(x, i, v, s)
    ctx.distill_bwd(x, i, v, keep, s, x)


# The C entry points: a context that is only an address, arguments that are wrong one at a time.  Nothing is launched.
FAKE = ctypes.create_string_buffer(4096)
HANDLE = ctypes.cast(FAKE, ctypes.c_void_p)
A = 1 << 20   # an aligned address that is never read


class NormFwdDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "weight", "bias_vec", "h", "y", "d_mean", "d_rstd", "y8", "d_bias_in", "d_amax",
                                               "d_bias_out")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "ld_x", "ld_residual", "ld_h", "ld_y")] + \
               [(n, ctypes.c_int32) for n in ("kind", "dt", "w_dt", "conv", "margin")] + [("eps", ctypes.c_float)]


class NormBwdDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dy", "h", "dh", "weight", "d_mean", "d_rstd", "dx", "dw", "db", "d_amax")] + \
               [(n, ctypes.c_int64) for n in ("rows", "cols", "ld_dy", "ld_h", "ld_dh", "ld_dx")] + \
               [(n, ctypes.c_int32) for n in ("kind", "dt", "w_dt", "reserved")]


def test_the_binding_packs_the_structures():
    assert fp8lin._NORM_FWD.size == ctypes.sizeof(NormFwdDesc) and fp8lin._NORM_BWD.size == ctypes.sizeof(NormBwdDesc)


def norm_fwd(ctx=HANDLE, **change):
    d = NormFwdDesc(x=A, residual=A, weight=A, bias_vec=A, h=A, y=A, d_mean=A, d_rstd=A, y8=A, d_bias_in=None, d_amax=A, d_bias_out=A,
                    rows=4, cols=32, ld_x=32, ld_residual=32, ld_h=32, ld_y=32, kind=0, dt=0, w_dt=0, conv=0, margin=0, eps=1e-5)
    for k, v in change.items():
        setattr(d, k, v)
    return fp8lin._lib.fp8_norm_fwd(ctx, bytes(d), None)


def norm_bwd(ctx=HANDLE, **change):
    d = NormBwdDesc(dy=A, h=A, dh=A, weight=A, d_mean=A, d_rstd=A, dx=A, dw=A, db=A, d_amax=A, rows=4, cols=32, ld_dy=32, ld_h=32,
                    ld_dh=32, ld_dx=32, kind=0, dt=0, w_dt=0, reserved=0)
    for k, v in change.items():
        setattr(d, k, v)
    return fp8lin._lib.fp8_norm_bwd(ctx, bytes(d), None)


E = fp8lin


@pytest.mark.parametrize("change,status", [
    (dict(ctx=None), E.ERR_NULL), (dict(x=None), E.ERR_NULL), (dict(d_bias_out=None), E.ERR_NULL), (dict(d_mean=None), E.ERR_NULL),
    (dict(d_rstd=None), E.ERR_NULL), (dict(h=None, y=None, d_mean=None, d_rstd=None, y8=None, d_amax=None, d_bias_out=None), E.ERR_NULL),
    (dict(rows=0), E.ERR_SHAPE), (dict(cols=0), E.ERR_SHAPE), (dict(cols=(1 << 30) + 1, ld_x=1 << 31), E.ERR_SHAPE), (dict(ld_x=31), E.ERR_SHAPE),
    (dict(ld_h=31), E.ERR_SHAPE), (dict(ld_y=31), E.ERR_SHAPE), (dict(ld_residual=31), E.ERR_SHAPE), (dict(eps=-1.0), E.ERR_SHAPE),
    (dict(eps=float("nan")), E.ERR_SHAPE), (dict(eps=float("inf")), E.ERR_SHAPE), (dict(kind=2), E.ERR_DTYPE), (dict(dt=3), E.ERR_DTYPE),
    (dict(conv=2), E.ERR_DTYPE), (dict(w_dt=-1), E.ERR_DTYPE), (dict(w_dt=1), E.ERR_UNSUPPORTED), (dict(dt=2, w_dt=0), E.ERR_UNSUPPORTED),
    (dict(x=A + 1), E.ERR_ALIGN), (dict(dt=2, w_dt=2, y=A + 2), E.ERR_ALIGN), (dict(d_amax=A + 2), E.ERR_ALIGN), (dict(weight=A + 1), E.ERR_ALIGN)])
def test_library_refuses_norm_forward(change, status):
    assert norm_fwd(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(ctx=None), E.ERR_NULL), (dict(dy=None), E.ERR_NULL), (dict(h=None), E.ERR_NULL), (dict(d_mean=None), E.ERR_NULL), (dict(d_rstd=None), E.ERR_NULL),
    (dict(dx=None, dw=None, db=None, d_amax=None), E.ERR_NULL), (dict(dx=None), E.ERR_NULL), (dict(rows=0), E.ERR_SHAPE), (dict(ld_dy=31), E.ERR_SHAPE),
    (dict(ld_h=31), E.ERR_SHAPE), (dict(ld_dh=31), E.ERR_SHAPE), (dict(ld_dx=31), E.ERR_SHAPE), (dict(kind=-1), E.ERR_DTYPE), (dict(w_dt=3), E.ERR_DTYPE),
    (dict(w_dt=1), E.ERR_UNSUPPORTED), (dict(dw=A + 1), E.ERR_ALIGN), (dict(dh=A + 1), E.ERR_ALIGN),
    (dict(cols=(1 << 22) + 1, ld_dy=1 << 23, ld_h=1 << 23, ld_dh=1 << 23, ld_dx=1 << 23), E.ERR_SHAPE)])
def test_library_refuses_norm_backward(change, status):
    assert norm_bwd(**change) == status


def call(name, order, change):
    args = dict(ctx=HANDLE, logits=A, dt=0, ld=100, rows=4, vocab=100, scale=1.0, targets=A, it=1, logprob=A, entropy=A, lse=A, saved=A, top_k=3,
                top_logprob=A, top_index=A, g=A, g_stride=1, g2=A, g2_stride=1, dx=A, ld_d=100, amax=A, index=A, ld_index=8, value=A, ld_value=8,
                listed=8, mode=1, loss=A, stream=None)
    args.update(change)
    return getattr(fp8lin._lib, name)(*[args[k] for k in order.split()])


HEAD = "ctx logits dt ld rows vocab scale "
LIST = "index it ld_index value ld_value listed mode "
CALLS = {"fp8_token_logprobs": HEAD + "targets it logprob entropy lse saved top_k top_logprob top_index stream",
         "fp8_token_logprobs_bwd": HEAD + "targets it saved g g_stride g2 g2_stride dx ld_d amax stream",
         "fp8_distill_fwd": HEAD + LIST + "loss saved stream",
         "fp8_distill_bwd": HEAD + LIST + "saved g g_stride dx ld_d amax stream"}


@pytest.mark.parametrize("name", CALLS)
def test_library_refuses_logits(name):
    for change, status in ((dict(ctx=None), E.ERR_NULL), (dict(logits=None), E.ERR_NULL), (dict(dt=3), E.ERR_DTYPE), (dict(it=2), E.ERR_DTYPE),
                           (dict(rows=0), E.ERR_SHAPE), (dict(rows=1 << 31), E.ERR_SHAPE), (dict(vocab=0), E.ERR_SHAPE), (dict(ld=99), E.ERR_SHAPE),
                           (dict(scale=0.0), E.ERR_SHAPE), (dict(scale=-1.0), E.ERR_SHAPE), (dict(scale=float("nan")), E.ERR_SHAPE),
                           (dict(scale=3e38), E.ERR_SHAPE), (dict(logits=A + 1), E.ERR_ALIGN), (dict(saved=A + 4), E.ERR_ALIGN)):
        assert call(name, CALLS[name], change) == status, change


@pytest.mark.parametrize("name,change,status", [
    ("fp8_token_logprobs", dict(targets=None), E.ERR_NULL), ("fp8_token_logprobs", dict(top_logprob=None), E.ERR_NULL),
    ("fp8_token_logprobs", dict(top_index=None), E.ERR_NULL), ("fp8_token_logprobs", dict(top_k=-1), E.ERR_SHAPE),
    ("fp8_token_logprobs", dict(top_k=101), E.ERR_SHAPE), ("fp8_token_logprobs", dict(top_k=129, vocab=200, ld=200), E.ERR_UNSUPPORTED),
    ("fp8_token_logprobs", dict(logprob=None, entropy=None, lse=None, saved=None, top_k=0), E.ERR_NULL),
    ("fp8_token_logprobs", dict(targets=A + 4), E.ERR_ALIGN), ("fp8_token_logprobs", dict(top_index=A + 4), E.ERR_ALIGN),
    ("fp8_token_logprobs_bwd", dict(saved=None), E.ERR_NULL), ("fp8_token_logprobs_bwd", dict(dx=None), E.ERR_NULL),
    ("fp8_token_logprobs_bwd", dict(g=None, g2=None), E.ERR_NULL), ("fp8_token_logprobs_bwd", dict(targets=None), E.ERR_NULL),
    ("fp8_token_logprobs_bwd", dict(ld_d=99), E.ERR_SHAPE), ("fp8_token_logprobs_bwd", dict(g_stride=-1), E.ERR_SHAPE),
    ("fp8_token_logprobs_bwd", dict(dx=A + 1), E.ERR_ALIGN),
    ("fp8_distill_fwd", dict(loss=None), E.ERR_NULL), ("fp8_distill_bwd", dict(g=None), E.ERR_NULL), ("fp8_distill_bwd", dict(saved=None), E.ERR_NULL),
    ("fp8_distill_bwd", dict(ld_d=99), E.ERR_SHAPE), ("fp8_distill_bwd", dict(dx=A + 1), E.ERR_ALIGN)])
def test_library_refuses(name, change, status):
    assert call(name, CALLS[name], change) == status


@pytest.mark.parametrize("name", ["fp8_distill_fwd", "fp8_distill_bwd"])
def test_library_refuses_lists(name):
    for change, status in ((dict(index=None), E.ERR_NULL), (dict(value=None), E.ERR_NULL), (dict(mode=2), E.ERR_DTYPE), (dict(listed=0), E.ERR_SHAPE),
                           (dict(ld_index=7), E.ERR_SHAPE), (dict(ld_value=7), E.ERR_SHAPE), (dict(listed=257, ld_index=257, ld_value=257), E.ERR_UNSUPPORTED),
                           (dict(vocab=(1 << 20) + 1, ld=1 << 21, ld_d=1 << 21), E.ERR_UNSUPPORTED), (dict(index=A + 4), E.ERR_ALIGN),
                           (dict(value=A + 2), E.ERR_ALIGN)):
        assert call(name, CALLS[name], change) == status, change


def test_library_refuses_other_distances_in_place():
    """An output in an input's place lies as the input does (one row has no distance)."""
    B = 1 << 24
    assert norm_fwd(residual=B, ld_x=40) == E.ERR_SHAPE and norm_fwd(x=B, ld_residual=40) == E.ERR_SHAPE
    assert norm_bwd(dh=B, ld_dy=40) == E.ERR_SHAPE and norm_bwd(dy=B, ld_dh=40) == E.ERR_SHAPE
    assert call("fp8_token_logprobs_bwd", CALLS["fp8_token_logprobs_bwd"], dict(ld=104)) == E.ERR_SHAPE
    assert call("fp8_distill_bwd", CALLS["fp8_distill_bwd"], dict(ld=104)) == E.ERR_SHAPE
