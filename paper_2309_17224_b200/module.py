"""``Fp8Linear``: a drop-in ``torch.nn.Linear`` whose three matmuls run in FP8.

The layer the paper describes (Section 2: Fig. 3b, Eq. 1-3 and Section 2.2 for
the backward pass; Section 3 for the two ways of choosing the scaling bias;
Section 3.1 for inference on weights quantised once), wired into autograd.
Everything numeric happens in the C-ABI library: this file allocates buffers,
keeps the per-tensor device scalars (amax and scaling bias of W, X and dY) and
marshals arguments.  The one exception is the gradient of the optional additive
bias vector, which the paper's layer does not have: it is ``dY.sum(0)`` in torch.

Scaling policies (``scaling=``):

``"amax"``      FP8-AMAX, just in time (Eq. 3): every tensor is quantised under
                the bias of its own current amax (two passes over the tensor).
``"predicted"`` FP8-AMAX in one pass: each tensor is cast under the bias its
                previous step left behind while its amax is taken; where Eq. 3
                gives another bias the cast is repeated.  Same bits as "amax".
``"constant"``  FP8-CSCALE (Section 3): the caller's constant biases
                (``constant_bias=(b_w, b_x, b_g)``), no amax at all.

``margin`` (Section 3.2) is subtracted from the gradient's bias.  In ``eval()``
mode the weight is quantised once and cached until ``train()`` is called again
or ``requantise()`` is asked for (post-training quantisation); activations of at
most 64 KB are then quantised inside the matmul's own launch.

``Norm`` and ``Fp8NormLinear`` put the decoder's norm in front of it (``include/fp8_norm.h``): the residual sum, layer norm or
its root-mean-square form, and, in the second, the linear whose FP8 input the norm writes itself.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import fp8lin

_W, _X, _G = 0, 1, 2
_default_ctx = {}


def default_context(device: int) -> "fp8lin.Context":
    """One library context per device, created on first use (it owns the split-contraction workspace)."""
    if device not in _default_ctx:
        _default_ctx[device] = fp8lin.Context(device)
    return _default_ctx[device]


def _out_dtype(dt):
    """The library writes bf16 or fp32: fp16 tensors get bf16 results."""
    return dt if dt in (torch.bfloat16, torch.float32) else torch.bfloat16


def _backward_matmuls(layer, g8, x8, w8, b_fwd, dx_dtype, want_dw):
    """(dX [T, K] of ``dx_dtype``, or None without one; dW in the weight's type, or None) from the FP8 bytes of a step."""
    lib, bg, (T, N), K = layer.ctx, layer.bias_words[_G:_G + 1], g8.shape, layer.in_features
    dx = dw = None
    if dx_dtype is not None:
        dx = torch.empty((T, K), dtype=dx_dtype, device=g8.device)
    if want_dw:
        dw = torch.empty((N, K), dtype=_out_dtype(layer.weight.dtype), device=g8.device)
    if dx is not None and dw is not None:
        # the two backward matmuls share dY8 and do not depend on each other (Section 2.2): one launch
        lib.linear_group([(fp8lin.MATMUL_DGRAD, g8, bg, w8, b_fwd[_W:_W + 1], dx),
                          (fp8lin.MATMUL_WGRAD, g8, bg, x8, b_fwd[_X:_X + 1], dw)], conv=layer.conv)
    elif dx is not None:
        lib.linear_dgrad(g8, bg, w8, None, b_fwd[_W:_W + 1], dx, conv=layer.conv)
    elif dw is not None:
        lib.linear_wgrad(g8, None, bg, x8, None, b_fwd[_X:_X + 1], dw, T, conv=layer.conv)
    if dw is not None and dw.dtype != layer.weight.dtype:
        dw = dw.to(layer.weight.dtype)
    return dx, dw


class _Fp8LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(fn, x, weight, bias_vec, layer):
        lib = layer.ctx
        K, N = layer.in_features, layer.out_features
        x2 = x.reshape(-1, K)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        T = x2.shape[0]
        dev = x2.device
        x8 = torch.empty((T, K), dtype=torch.uint8, device=dev)
        y = torch.empty((T, N), dtype=layer.out_dtype or _out_dtype(x.dtype), device=dev)
        am, bi = layer.amax, layer.bias_words
        if layer.training and layer.scaling != "constant" and T > 128:
            # training: W and X are quantised together, all passes of both tensors in two launches (fp8_cast_group)
            w8 = torch.empty((N, K), dtype=torch.uint8, device=dev)
            lib.cast_group([(fp8lin.E4, weight.detach(), am[_W:_W + 1], bi[_W:_W + 1], w8),
                            (fp8lin.E4, x2, am[_X:_X + 1], bi[_X:_X + 1], x8)], conv=layer.conv,
                           predicted=layer.scaling == "predicted")
            lib.linear_fwd(x8, bi[_X:_X + 1], w8, bi[_W:_W + 1], y, bias_vec=bias_vec, conv=layer.conv)
            fn.layer, fn.x_shape, fn.has_bias = layer, x.shape, bias_vec is not None
            fn.save_for_backward(x8, w8, bi[:2].clone())
            return y.reshape(*x.shape[:-1], N)
        w8, w8_is_old = layer._quantised_weight(weight)
        # the inference calls may read the weight's bytes early: only once those were written by an earlier forward pass
        frozen = (not layer.training) and w8_is_old
        if frozen and layer.scaling != "constant" and T <= 128:
            # inference on a few rows: the activation is quantised by the matmul's own launch where it is small enough
            lib.linear_infer_cast(x2, am[_X:_X + 1], bi[_X:_X + 1], x8, w8, bi[_W:_W + 1], y, bias_vec=bias_vec,
                                  conv=layer.conv)
        else:
            layer._quantise(fp8lin.E4, x2, _X, x8, margin=0)
            run = lib.linear_infer if frozen else lib.linear_fwd
            run(x8, bi[_X:_X + 1], w8, bi[_W:_W + 1], y, bias_vec=bias_vec, conv=layer.conv)
        fn.layer = layer
        fn.x_shape = x.shape
        fn.has_bias = bias_vec is not None
        # X8 and W8 are cast once in the forward pass and used again by the backward matmuls (Section 2.2); their
        # biases are copied because the layer's words are rewritten by its next forward pass
        fn.save_for_backward(x8, w8, bi[:2].clone())
        return y.reshape(*x.shape[:-1], N)

    @staticmethod
    def backward(fn, dy):
        layer = fn.layer
        N = layer.out_features
        x8, w8, b_fwd = fn.saved_tensors
        T = x8.shape[0]
        dy2 = dy.reshape(T, N)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        g8 = torch.empty((T, N), dtype=torch.uint8, device=dy2.device)
        layer._quantise(fp8lin.E5, dy2, _G, g8, margin=layer.margin)
        dx, dw = _backward_matmuls(layer, g8, x8, w8, b_fwd, _out_dtype(dy.dtype) if fn.needs_input_grad[0] else None,
                                   fn.needs_input_grad[1])
        db = None
        if dx is not None:
            dx = dx.reshape(fn.x_shape)
        if fn.has_bias and fn.needs_input_grad[2]:
            db = dy2.sum(0, dtype=torch.float32).to(layer.bias.dtype)   # not part of the paper's layer
        return dx, dw, db, None


class Fp8Linear(torch.nn.Module):
    """``y = x W^T (+ b)`` with X, W quantised to E4 and dY to E5 under per-tensor power-of-two scaling biases.

    weight: [out_features, in_features], bf16 (default) or fp32 master weights (the cast reads either); inputs and
    output gradients bf16, fp16 or fp32; outputs and gradients bf16 or fp32 (fp16 is not an output type of the
    library).  ``in_features`` must be a multiple of 16 (rows of FP8 bytes are fetched in 16-byte units).
    After a backward pass ``amax`` and ``bias_words`` hold the three tensors' statistics of that step
    (order W, X, dY), on the device; nothing here synchronises with the host."""

    def __init__(self, in_features: int, out_features: int, bias: bool = False, device="cuda", dtype=torch.bfloat16,
                 scaling: str = "amax", margin: int = 0, conv: int = fp8lin.CONV_PAPER,
                 constant_bias: Optional[Sequence[int]] = None, out_dtype=None, ctx: Optional["fp8lin.Context"] = None):
        super().__init__()
        if scaling not in ("amax", "predicted", "constant"):
            raise ValueError("scaling must be 'amax', 'predicted' or 'constant'")
        if scaling == "constant" and (constant_bias is None or len(constant_bias) != 3):
            raise ValueError("scaling='constant' needs constant_bias=(b_w, b_x, b_g)")
        if in_features % 16:
            raise ValueError("in_features must be a multiple of 16")
        dev = torch.device(device)
        self.in_features, self.out_features = in_features, out_features
        self.scaling, self.margin, self.conv, self.out_dtype = scaling, int(margin), conv, out_dtype
        self.ctx = ctx if ctx is not None else default_context(dev.index or 0)
        self.weight = torch.nn.Parameter(torch.empty((out_features, in_features), device=dev, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_features, device=dev, dtype=dtype)) if bias else None
        torch.nn.init.normal_(self.weight, std=0.02)
        self.register_buffer("amax", torch.zeros(3, dtype=torch.float32, device=dev), persistent=False)
        init = list(constant_bias) if scaling == "constant" else [0, 0, 0]
        self.register_buffer("bias_words", torch.tensor(init, dtype=torch.int32, device=dev), persistent=False)
        self._w8 = None            # FP8 bytes of the weight, kept while the module is in eval() mode
        self._w8_version = None

    # -- quantisation -----------------------------------------------------------------------------------------------
    def _quantise(self, fmt, t, which, out8, margin):
        c = self.ctx
        a, b = self.amax[which:which + 1], self.bias_words[which:which + 1]
        cast = c.cast_e4 if fmt == fp8lin.E4 else c.cast_e5
        if self.scaling == "constant":
            cast(t, b, conv=self.conv, y=out8)
        elif self.scaling == "predicted":
            c.cast_predicted(fmt, t, a, b, out8, conv=self.conv, margin=margin)
        else:
            cast(t, None, conv=self.conv, margin=margin, d_amax_out=a, d_bias_out=b, y=out8)

    def _quantised_weight(self, weight):
        if not self.training and self._w8 is not None and self._w8_version == weight._version:
            return self._w8, True
        w8 = torch.empty((self.out_features, self.in_features), dtype=torch.uint8, device=weight.device)
        w = weight.detach()
        if not self.training and self.scaling != "constant":
            # post-training quantisation (Section 3.1): amax, bias and bytes once
            self.ctx.ptq_weights(w, self.conv, w8, None, self.bias_words[_W:_W + 1], self.amax[_W:_W + 1])
        else:
            self._quantise(fp8lin.E4, w, _W, w8, margin=0)
        if not self.training:
            self._w8, self._w8_version = w8, weight._version
        return w8, False

    def requantise(self):
        """Forget the cached FP8 weight (eval mode): the next forward pass quantises the weight again."""
        self._w8 = self._w8_version = None

    def train(self, mode: bool = True):
        self.requantise()
        return super().train(mode)

    def forward(self, x):
        return _Fp8LinearFn.apply(x, self.weight, self.bias, self)

    def extra_repr(self):
        return (f"in_features={self.in_features}, out_features={self.out_features}, bias={self.bias is not None}, "
                f"scaling={self.scaling}, margin={self.margin}")


# -- the norm in front of a linear -----------------------------------------------------------------------------------------
_NORM_KINDS = {"layer": fp8lin.NORM_LAYER, "rms": fp8lin.NORM_RMS}


def matrix_rows(t, columns):
    """t as [rows, columns] with contiguous rows that do not overlap (gradients of sums and means are expanded numbers)."""
    t = t.reshape(-1, columns)
    plain = t.shape[0] <= 1 or t.stride(0) >= columns
    return t if plain and (columns == 1 or t.stride(1) == 1) else t.contiguous()


def _norm_rows(x, residual, features):
    """x and the residual as [rows, features] with contiguous rows."""
    if x.shape[-1] != features or (residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype)):
        raise ValueError(f"x [..., {features}] and a residual of its shape and type expected, got {tuple(x.shape)} {x.dtype}"
                         + ("" if residual is None else f" and {tuple(residual.shape)} {residual.dtype}"))
    return matrix_rows(x, features), None if residual is None else matrix_rows(residual, features)


def _norm_statistics(rows, kind, device):
    """Buffers of a forward pass: (mean or None, 1 / standard deviation)."""
    f32 = dict(dtype=torch.float32, device=device)
    return (torch.empty(rows, **f32) if kind == fp8lin.NORM_LAYER else None), torch.empty(rows, **f32)


def _norm_backward(layer, dy, h, weight, mean, rstd, dh, want_w, want_b):
    """(gradient of the sum, of the weight, of the additive vector) in h's and the weight's types."""
    dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    dw = torch.empty_like(weight) if want_w else None
    db = torch.empty_like(weight) if want_b else None
    if dh is not None:
        dh = matrix_rows(dh, h.shape[1])
    layer.ctx.norm_bwd(dy, h, weight, mean, rstd, dx, dh=dh, dw=dw, db=db, kind=layer.norm_kind)
    return dx, dw, db


class _NormFn(torch.autograd.Function):
    """(y, h); h is x itself where there is no residual (and then not an output)."""

    @staticmethod
    def forward(fn, x, residual, weight, bias, layer):
        x2, r2 = _norm_rows(x, residual, layer.features)
        h = x2 if r2 is None else torch.empty(x2.shape, dtype=x.dtype, device=x.device)
        y = torch.empty(x2.shape, dtype=x.dtype, device=x.device)
        mean, rstd = _norm_statistics(x2.shape[0], layer.norm_kind, x.device)
        layer.ctx.norm_fwd(x2, weight.detach(), None if bias is None else bias.detach(), residual=r2, eps=layer.eps, kind=layer.norm_kind,
                           h=None if r2 is None else h, y=y, d_mean=mean, d_rstd=rstd)
        fn.layer, fn.shape, fn.with_h = layer, x.shape, r2 is not None
        fn.set_materialize_grads(False)
        fn.save_for_backward(h, weight, mean, rstd)
        y = y.reshape(x.shape)
        return (y, h.reshape(x.shape)) if fn.with_h else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, dy, dh=None):
        h, weight, mean, rstd = fn.saved_tensors
        if dy is None:
            return dh, dh if fn.with_h else None, None, None, None
        dx, dw, db = _norm_backward(fn.layer, matrix_rows(dy, h.shape[1]), h, weight, mean, rstd, dh, fn.needs_input_grad[2],
                                    fn.needs_input_grad[3])
        dx = dx.reshape(fn.shape)
        return dx, dx if fn.with_h else None, dw, db, None


class Norm(torch.nn.Module):
    """Layer norm (``kind="layer"``, with an additive vector) or its root-mean-square form (``"rms"``) over the last dimension.

    ``forward(x)`` gives y; ``forward(x, residual)`` gives (y, x + residual), both from one call.  x bf16, fp16 or fp32, y of
    its type; weight and bias of that type or float32."""

    def __init__(self, features: int, kind: str = "layer", eps: float = 1e-5, device="cuda", dtype=torch.bfloat16,
                 ctx: Optional["fp8lin.Context"] = None):
        super().__init__()
        if kind not in _NORM_KINDS:
            raise ValueError("kind must be 'layer' or 'rms'")
        dev = torch.device(device)
        self.features, self.kind, self.norm_kind, self.eps = features, kind, _NORM_KINDS[kind], float(eps)
        self.ctx = ctx if ctx is not None else default_context(dev.index or 0)
        self.weight = torch.nn.Parameter(torch.ones(features, device=dev, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(features, device=dev, dtype=dtype)) if kind == "layer" else None

    def forward(self, x, residual=None):
        return _NormFn.apply(x, residual, self.weight, self.bias, self)

    def extra_repr(self):
        return f"{self.features}, kind={self.kind}, eps={self.eps}"


class _Fp8NormLinearFn(torch.autograd.Function):
    """(linear(norm(x + residual)), x + residual); the sum is an output only where there is a residual."""

    @staticmethod
    def forward(fn, x, residual, norm_weight, norm_bias, weight, bias_vec, layer):
        lib, K, N = layer.ctx, layer.in_features, layer.out_features
        x2, r2 = _norm_rows(x, residual, K)
        T, dev = x2.shape[0], x2.device
        h = x2 if r2 is None else torch.empty(x2.shape, dtype=x.dtype, device=dev)
        x8 = torch.empty((T, K), dtype=torch.uint8, device=dev)
        y = torch.empty((T, N), dtype=layer.out_dtype or _out_dtype(x.dtype), device=dev)
        mean, rstd = _norm_statistics(T, layer.norm_kind, dev)
        am, bi = layer.amax, layer.bias_words
        constant = layer.scaling == "constant"
        w8, w8_is_old = layer._quantised_weight(weight)
        lib.norm_fwd(x2, norm_weight.detach(), None if norm_bias is None else norm_bias.detach(), residual=r2, eps=layer.eps,
                     kind=layer.norm_kind, h=None if r2 is None else h, d_mean=mean, d_rstd=rstd, y8=x8,
                     d_bias=bi[_X:_X + 1] if constant else None, d_amax_out=None if constant else am[_X:_X + 1],
                     d_bias_out=None if constant else bi[_X:_X + 1], conv=layer.conv)
        run = lib.linear_infer if (not layer.training) and w8_is_old else lib.linear_fwd
        run(x8, bi[_X:_X + 1], w8, bi[_W:_W + 1], y, bias_vec=bias_vec, conv=layer.conv)
        fn.layer, fn.shape, fn.with_h, fn.has_bias = layer, x.shape, r2 is not None, bias_vec is not None
        fn.set_materialize_grads(False)
        fn.save_for_backward(h, norm_weight, mean, rstd, x8, w8, bi[:2].clone())
        y = y.reshape(*x.shape[:-1], N)
        return (y, h.reshape(x.shape)) if fn.with_h else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, dy, dh=None):
        layer = fn.layer
        h, norm_weight, mean, rstd, x8, w8, b_fwd = fn.saved_tensors
        if dy is None:
            return dh, dh if fn.with_h else None, None, None, None, None, None
        T, N = x8.shape[0], layer.out_features
        dy2 = dy.reshape(T, N)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        g8 = torch.empty((T, N), dtype=torch.uint8, device=dy2.device)
        layer._quantise(fp8lin.E5, dy2, _G, g8, margin=layer.margin)
        need = fn.needs_input_grad
        # the gradient of the norm's output has the sum's type (FP16: by way of FP32, the library writes no FP16)
        through = need[0] or need[1] or need[2] or need[3]
        dn, dw = _backward_matmuls(layer, g8, x8, w8, b_fwd, (torch.float32 if h.dtype == torch.float16 else h.dtype) if through else None,
                                   need[4])
        dx = d_norm_w = d_norm_b = db = None
        if through:
            dn = dn.to(h.dtype)
            dx, d_norm_w, d_norm_b = _norm_backward(layer, dn, h, norm_weight, mean, rstd, dh, need[2], need[3])
            dx = dx.reshape(fn.shape)
        if fn.has_bias and need[5]:
            db = dy2.sum(0, dtype=torch.float32).to(layer.bias.dtype)   # not part of the paper's layer
        return dx, dx if fn.with_h else None, d_norm_w, d_norm_b, dw, db, None


class Fp8NormLinear(Fp8Linear):
    """``Norm`` and ``Fp8Linear`` as one: the norm writes the FP8 bytes that the matmul reads, under the bias of their amax
    (``scaling="amax"``, Eq. 3 just in time) or a constant one, and its 16-bit output does not exist.

    ``forward(x)`` gives the linear's output, ``forward(x, residual)`` that and x + residual.  Parameters: those of
    ``Fp8Linear`` and ``norm_weight`` and, with ``kind="layer"``, ``norm_bias``."""

    def __init__(self, in_features: int, out_features: int, kind: str = "layer", eps: float = 1e-5, norm_dtype=None, device="cuda",
                 dtype=torch.bfloat16, scaling: str = "amax", **kw):
        if kind not in _NORM_KINDS:
            raise ValueError("kind must be 'layer' or 'rms'")
        if scaling == "predicted":
            raise ValueError("scaling must be 'amax' or 'constant': the norm has no bytes before its amax to guess for")
        super().__init__(in_features, out_features, device=device, dtype=dtype, scaling=scaling, **kw)
        self.kind, self.norm_kind, self.eps = kind, _NORM_KINDS[kind], float(eps)
        like = dict(device=self.weight.device, dtype=norm_dtype or dtype)
        self.norm_weight = torch.nn.Parameter(torch.ones(in_features, **like))
        self.norm_bias = torch.nn.Parameter(torch.zeros(in_features, **like)) if kind == "layer" else None

    def forward(self, x, residual=None):
        return _Fp8NormLinearFn.apply(x, residual, self.norm_weight, self.norm_bias, self.weight, self.bias, self)

    def extra_repr(self):
        return f"{super().extra_repr()}, kind={self.kind}, eps={self.eps}"
