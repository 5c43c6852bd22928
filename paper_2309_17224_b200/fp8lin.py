"""Python face of ``libfp8lin.so``: argument marshalling only.

Every function here has the name and the argument order of the C entry point
declared in ``include/fp8lin.h``; tensors are torch CUDA tensors whose
``data_ptr()`` is handed through, the stream is torch's current stream.  There
is no arithmetic and no fallback in this module: if the library is missing the
import fails, and a non-zero status raises ``Fp8Error``.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import c_int, c_int32, c_int64, c_uint, c_uint64, c_void_p, c_float, c_char_p, POINTER, byref

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfp8lin.so")

OK = 0
ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_DTYPE, ERR_UNSUPPORTED, ERR_CUDA, ERR_DEVICE_TIMEOUT, ERR_TOO_LARGE = range(1, 9)
E4, E5 = 0, 1
CONV_PAPER, CONV_NATIVE = 0, 1
BF16, F16, F32 = 0, 1, 2
GROUP_AMAX_CAST, GROUP_PREDICTED, GROUP_AMAX_ONLY, GROUP_CAST_ONLY = 0, 1, 2, 3
MM_FWD, MM_DGRAD, MM_WGRAD = 0, 1, 2
ACT_NONE = 0
ACT_GELU = 1
ACT_SWIGLU = 2
FLAG_NONFINITE_AMAX, FLAG_ZERO_AMAX, FLAG_SATURATED, FLAG_TIMEOUT, FLAG_BAD_INDEX = 1, 2, 4, 8, 16
KV_BIAS_NONFINITE, KV_BIAS_MAX = -128, 64
NORM_LAYER, NORM_RMS = 0, 1
I32, I64 = 0, 1
DISTILL_TOP, DISTILL_REST = 0, 1
LOSS_SAVED, LOSS_TOP_MAX, LOSS_LISTED_MAX, LOSS_VOCAB_MAX = 4, 128, 256, 1 << 20

SYMBOLS = (
    "fp8_create", "fp8_destroy", "fp8_status_string", "fp8_device_flags", "fp8_amax", "fp8_scaling_bias",
    "fp8_scaling_bias_host", "fp8_cast_e4", "fp8_cast_e5", "fp8_ptq_weights", "fp8_linear_fwd", "fp8_linear_dgrad",
    "fp8_linear_wgrad", "fp8_amax_noalloc", "fp8_linear_fwd_act", "fp8_cast_predicted", "fp8_prediction_stats",
    "fp8_linear_dgrad_act", "fp8_selftest_wait_expiry", "fp8_range_stats", "fp8_linear_fwd_q", "fp8_linear_dgrad_q", "fp8_amax_history_bias", "fp8_launch_count", "fp8_cast_group", "fp8_selftest_mma_ceiling", "fp8_bias_log_append", "fp8_bias_mode", "fp8_linear_f16acc", "fp8_linear_infer", "fp8_linear_infer_cast", "fp8_linear_group",
    "fp8_kv_append", "fp8_kv_read", "fp8_attn_paged",
    "fp8_norm_fwd", "fp8_norm_bwd", "fp8_token_logprobs", "fp8_token_logprobs_bwd", "fp8_distill_fwd", "fp8_distill_bwd",
    "fp8h_gelu", "fp8h_gelu_backward", "fp8h_mse_grad", "fp8h_sgd",
)

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2309_17224_b200.build` "
        "(there is no fallback implementation)")

_lib = ctypes.CDLL(LIB_PATH)

_P = c_void_p
_lib.fp8_create.argtypes = [POINTER(c_void_p), c_int]
_lib.fp8_destroy.argtypes = [_P]
_lib.fp8_status_string.argtypes = [c_int]
_lib.fp8_status_string.restype = c_char_p
_lib.fp8_device_flags.argtypes = [_P, _P, POINTER(c_uint), c_int]
_lib.fp8_selftest_wait_expiry.argtypes = [_P, ctypes.c_uint64, _P]
_lib.fp8_selftest_mma_ceiling.argtypes = [_P, _P, _P, c_int64, c_int64, c_int64, _P]
_lib.fp8_bias_log_append.argtypes = [_P, _P, c_int32, _P, c_int32, c_int32, _P, _P, c_int32, _P]
_lib.fp8_bias_mode.argtypes = [_P, _P, c_int32, _P, c_int32, c_int32, c_int32, _P, _P, _P, _P]
_lib.fp8_amax.argtypes = [_P, _P, c_int, c_int64, c_int64, c_int64, _P, _P]
_lib.fp8_amax_noalloc.argtypes = [_P, c_int, c_int64, c_int64, c_int64, _P, _P]
_lib.fp8_scaling_bias.argtypes = [_P, _P, c_int, c_int, c_int32, _P, _P]
_lib.fp8_scaling_bias_host.argtypes = [c_float, c_int, c_int, c_int32, POINTER(c_int32)]
_cast_args = [_P, _P, c_int, c_int64, c_int64, c_int64, _P, c_int, c_int32, _P, _P, _P, _P, _P]
_lib.fp8_cast_e4.argtypes = _cast_args
_lib.fp8_cast_e5.argtypes = _cast_args
_lib.fp8_cast_predicted.argtypes = [_P, c_int, _P, c_int, c_int64, c_int64, c_int64, c_int, c_int32, _P, _P, _P, _P]
_lib.fp8_prediction_stats.argtypes = [_P, _P, POINTER(c_uint), POINTER(c_uint), c_int]
_lib.fp8_range_stats.argtypes = [_P, c_int, _P, c_int, c_int64, c_int64, c_int64, _P, c_int, _P, _P]
_lib.fp8_ptq_weights.argtypes = [_P, _P, c_int, c_int64, c_int64, c_int64, c_int, _P, _P, _P, _P, _P]
_lib.fp8_linear_fwd.argtypes = [_P, _P, _P, _P, _P, _P, c_int, _P, c_int, _P, c_int64, c_int64, c_int64, c_int, _P]
_lib.fp8_linear_infer.argtypes = _lib.fp8_linear_fwd.argtypes
_lib.fp8_linear_infer_cast.argtypes = [_P, _P, c_int, c_int, _P, _P, _P, _P, _P, _P, c_int, _P, c_int, _P, c_int64, c_int64,
                                       c_int64, c_int, _P]
_lib.fp8_linear_fwd_act.argtypes = [_P, _P, _P, _P, _P, _P, c_int, _P, _P, c_int, _P, c_int64, c_int64, c_int64, c_int, _P]
_lib.fp8_linear_dgrad.argtypes = [_P, _P, _P, _P, _P, _P, _P, c_int, _P, c_int64, c_int64, c_int64, c_int, _P]
_lib.fp8_linear_dgrad_act.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, _P, c_int, _P, c_int64, c_int64, c_int64, c_int, _P]
_lib.fp8_amax_history_bias.argtypes = [_P, _P, c_int32, _P, _P, c_int, c_int, c_int32, _P, _P]
_lib.fp8_linear_fwd_q.argtypes = [_P, _P, _P, _P, _P, _P, c_int, c_int, _P, _P, _P, _P, _P, c_int64, c_int64, c_int64,
                                  c_int, _P]
_lib.fp8_linear_dgrad_q.argtypes = [_P, _P, _P, _P, _P, _P, c_int, _P, _P, _P, _P, _P, _P, c_int64, c_int64, c_int64,
                                    c_int, _P]
_lib.fp8_linear_f16acc.argtypes = [_P, c_int, _P, _P, _P, _P, _P, c_int, c_int32, c_int64, c_int64, c_int64, c_int, _P]
_lib.fp8_linear_wgrad.argtypes = [_P, _P, _P, _P, _P, _P, _P, _P, c_int, c_int64, c_int64, c_int64, c_int, _P]


class GroupItem(ctypes.Structure):
    """``fp8_group_item_t``."""
    _fields_ = [("x", c_void_p), ("x_dt", c_int), ("rows", c_int64), ("cols", c_int64), ("ld", c_int64),
                ("fmt", c_int), ("margin", c_int32), ("d_amax", c_void_p), ("d_bias", c_void_p), ("y", c_void_p)]


_lib.fp8_cast_group.argtypes = [_P, POINTER(GroupItem), c_int32, c_int, c_int32, _P]


class MatmulItem(ctypes.Structure):
    """``fp8_matmul_item_t``."""
    _fields_ = [("kind", c_int32), ("bias_dt", c_int32), ("a8", c_void_p), ("d_ba", c_void_p), ("b8", c_void_p),
                ("d_bb", c_void_p), ("bias_vec", c_void_p), ("out", c_void_p), ("d_amax_out", c_void_p),
                ("out_dt", c_int32), ("reserved", c_int32), ("T", c_int64), ("K", c_int64), ("N", c_int64)]


_lib.fp8_linear_group.argtypes = [_P, POINTER(MatmulItem), c_int32, c_int, _P]


class KvCacheDesc(ctypes.Structure):
    """``fp8_kv_cache_t``."""
    _fields_ = [("k8", c_void_p), ("v8", c_void_p), ("bk", c_void_p), ("bv", c_void_p), ("page_stride", c_int64),
                ("bias_stride", c_int64), ("pages", c_int32), ("kv_heads", c_int32), ("page_size", c_int32),
                ("head_dim", c_int32)]


class SeqBatchDesc(ctypes.Structure):
    """``fp8_seq_batch_t``."""
    _fields_ = [("d_q_start", c_void_p), ("d_kv_len", c_void_p), ("d_page_table", c_void_p), ("table_stride", c_int64),
                ("seqs", c_int32), ("tokens", c_int32), ("max_q_len", c_int32), ("max_kv_len", c_int32)]


_lib.fp8_kv_append.argtypes = [_P, POINTER(KvCacheDesc), POINTER(SeqBatchDesc), _P, _P, c_int, c_int64, c_int64, c_int, _P]
_lib.fp8_kv_read.argtypes = _lib.fp8_kv_append.argtypes
_lib.fp8_attn_paged.argtypes = [_P, POINTER(KvCacheDesc), POINTER(SeqBatchDesc), _P, c_int64, c_int32, _P, c_int64, _P,
                                c_float, c_int32, c_int, _P]


# ``fp8_norm_fwd_t`` and ``fp8_norm_bwd_t``, field by field (packing is several times quicker than a ctypes.Structure)
_NORM_FWD = struct.Struct("@12P6q5if")
_NORM_BWD = struct.Struct("@10P6q4i")

_lib.fp8_norm_fwd.argtypes = [_P, c_char_p, _P]
_lib.fp8_norm_bwd.argtypes = [_P, c_char_p, _P]
_logits_args = [_P, _P, c_int, c_int64, c_int64, c_int64, c_float]
_list_args = [_P, c_int, c_int64, _P, c_int64, c_int32, c_int]
_lib.fp8_token_logprobs.argtypes = _logits_args + [_P, c_int, _P, _P, _P, _P, c_int32, _P, _P, _P]
_lib.fp8_token_logprobs_bwd.argtypes = _logits_args + [_P, c_int, _P, _P, c_int64, _P, c_int64, _P, c_int64, _P, _P]
_lib.fp8_distill_fwd.argtypes = _logits_args + _list_args + [_P, _P, _P]
_lib.fp8_distill_bwd.argtypes = _logits_args + _list_args + [_P, _P, c_int64, _P, c_int64, _P, _P]
_lib.fp8h_gelu.argtypes = [_P, _P, c_int64, _P]
_lib.fp8h_gelu_backward.argtypes = [_P, _P, _P, c_int64, _P]
_lib.fp8h_mse_grad.argtypes = [_P, _P, ctypes.c_float, _P, c_int64, _P]
_lib.fp8h_sgd.argtypes = [_P, _P, ctypes.c_float, _P, c_int64, _P]
for _name in SYMBOLS:
    if _name != "fp8_status_string":
        getattr(_lib, _name).restype = c_int


class Fp8Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def status_string(status: int) -> str:
    return _lib.fp8_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise Fp8Error(status, where)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream():
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream(device):
    """The current stream's handle without the stream object (calls of a few microseconds notice the difference)."""
    return torch._C._cuda_getCurrentRawStream(device)


_DT = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}


def _ld(x):
    """Leading dimension of a 2-D tensor (torch leaves the stride of a size-1 dimension arbitrary)."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def launch_count() -> int:
    """Kernels this library has launched in this process so far."""
    out = c_uint64(0)
    _check(_lib.fp8_launch_count(byref(out)), "fp8_launch_count")
    return out.value


def scaling_bias_host(amax: float, fmt: int, conv: int = CONV_PAPER, margin: int = 0) -> int:
    out = c_int32(0)
    _check(_lib.fp8_scaling_bias_host(c_float(amax), fmt, conv, margin, byref(out)), "fp8_scaling_bias_host")
    return out.value


def amax_noalloc(x, d_amax, rows=None, cols=None, ld=None):
    """``fp8_amax_noalloc``: amax without a context and without any device
    allocation by the library (for callers that own all device memory or may
    not call cudaMalloc).  Contiguous bf16 input of at most 2^29 elements;
    calls on one device must not overlap on the GPU."""
    rows = x.shape[0] if rows is None else rows
    cols = x.shape[1] if cols is None else cols
    ld = _ld(x) if ld is None else ld
    _check(_lib.fp8_amax_noalloc(_ptr(x), _DT[x.dtype], rows, cols, ld, _ptr(d_amax), _stream()), "fp8_amax_noalloc")


def group_items(tensors):
    """A ctypes array of ``fp8_group_item_t`` from (fmt, x, d_amax, d_bias, y[, margin]) tuples; build it once
    and hand it to ``Context.cast_group`` every step (the tensors must stay alive)."""
    arr = (GroupItem * len(tensors))()
    for it, t in zip(arr, tensors):
        fmt, x, d_amax, d_bias, y = t[:5]
        it.x, it.x_dt, it.rows, it.cols, it.ld = x.data_ptr(), _DT[x.dtype], x.shape[0], x.shape[1], _ld(x)
        it.fmt, it.margin = fmt, (t[5] if len(t) > 5 else 0)
        it.d_amax = d_amax.data_ptr() if d_amax is not None else None
        it.d_bias, it.y = d_bias.data_ptr(), (y.data_ptr() if y is not None else None)
    return arr


class KvCache:
    """The pages of one layer's cache (``fp8_kv_cache_t``): k8, v8 uint8 [pages, kv_heads, page_size, head_dim], bk, bv
    int8 [pages, kv_heads, page_size].  The first dimension may be strided (keys and values of a page in one buffer)."""

    def __init__(self, k8, v8, bk, bv, conv=CONV_PAPER):
        pages, heads, size, dim = k8.shape
        for t, shape, dt in ((k8, k8.shape, torch.uint8), (v8, k8.shape, torch.uint8), (bk, k8.shape[:3], torch.int8),
                             (bv, k8.shape[:3], torch.int8)):
            if t.shape != shape or t.dtype != dt or not t[0].is_contiguous() or not t.is_cuda:
                raise ValueError("k8, v8: uint8 [pages, kv_heads, page_size, head_dim]; bk, bv: int8 [pages, kv_heads, "
                                 "page_size]; on the GPU, each page contiguous")
        self.device = k8.get_device()
        if any(t.get_device() != self.device for t in (v8, bk, bv)):
            raise ValueError("k8, v8, bk and bv on one GPU")
        if _page_stride(k8) != _page_stride(v8) or _page_stride(bk) != _page_stride(bv):
            raise ValueError("k8 and v8, bk and bv have their pages equally far apart")
        self.k8, self.v8, self.bk, self.bv, self.conv = k8, v8, bk, bv, conv
        self.kv_heads, self.page_size, self.head_dim = heads, size, dim
        self._desc = KvCacheDesc(k8.data_ptr(), v8.data_ptr(), bk.data_ptr(), bv.data_ptr(), _page_stride(k8),
                                 _page_stride(bk), pages, heads, size, dim)
        self._ref = byref(self._desc)


def _page_stride(t):
    return t.stride(0) if t.shape[0] > 1 else t[0].numel()


class SeqBatch:
    """The sequences of one call (``fp8_seq_batch_t``): q_start int32 [seqs + 1], kv_len int32 [seqs], page_table int32
    [seqs, table width], all on the GPU; the bounds of rows and tokens per sequence are host numbers.  Every row of the table
    has a column for each page of max_kv_len tokens (checked by the calls, which know the page size)."""

    def __init__(self, q_start, kv_len, page_table, max_q_len, max_kv_len):
        seqs = kv_len.shape[0]
        for t in (q_start, kv_len, page_table):
            if t.dtype != torch.int32 or (t.shape[-1] > 1 and t.stride(-1) != 1) or not t.is_cuda:
                raise ValueError("q_start, kv_len and page_table are int32 tensors on the GPU")
        if q_start.shape != (seqs + 1,) or kv_len.dim() != 1 or page_table.dim() != 2 or page_table.shape[0] != seqs:
            raise ValueError("q_start [seqs + 1], kv_len [seqs], page_table [seqs, width]")
        self.device = q_start.get_device()
        if kv_len.get_device() != self.device or page_table.get_device() != self.device:
            raise ValueError("q_start, kv_len and page_table on one GPU")
        self.q_start, self.kv_len, self.page_table = q_start, kv_len, page_table
        self._width, self._max_kv_len = page_table.shape[1], max_kv_len
        self._desc = SeqBatchDesc(q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(),
                                  page_table.stride(0) if seqs > 1 else self._width, seqs, 0, max_q_len, max_kv_len)
        self._ref = byref(self._desc)
        self._by_tokens = {}

    def _of(self, tokens):
        """The descriptor for a call on that many rows.  Calls change no descriptor, so threads can share a batch."""
        ref = self._by_tokens.get(tokens)
        if ref is None:
            desc = SeqBatchDesc.from_buffer_copy(self._desc)
            desc.tokens = tokens
            ref = self._by_tokens.setdefault(tokens, byref(desc))
        return ref


def _check_handles(cache, batch, device):
    if cache.device != device or batch.device != device:
        raise ValueError(f"cache and batch on the context's GPU {device} expected")
    # the library sees the distance between the table's rows only: in a slice of a wider table that is more than a row has
    if batch._width * cache.page_size < batch._max_kv_len:
        raise ValueError(f"page_table has {batch._width} columns of {cache.page_size} tokens, max_kv_len is {batch._max_kv_len}")


def _rows3(t, heads, dim, what, device):
    """Check a [tokens, heads, head_dim] tensor on the context's GPU whose heads are contiguous; its row distance in
    elements."""
    shape, stride = t.shape, t.stride()
    if t.get_device() != device:
        raise ValueError(f"{what}: a tensor on GPU {device} expected, got one on {t.device}")
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or stride[2] != 1 or (heads > 1 and stride[1] != dim):
        raise ValueError(f"{what}: [tokens, {heads}, {dim}] with contiguous heads expected, got {tuple(shape)} "
                         f"strides {stride}")
    return stride[0] if shape[0] > 1 else heads * dim


_IT = {torch.int32: I32, torch.int64: I64}


def _matrix(t, shape, dtypes, what, device):
    """Check a 2-D tensor (shape, one of the types, contiguous rows, the context's GPU); its row distance in elements."""
    own = t.shape
    if t.get_device() == device and t.dtype in dtypes and len(own) == 2 and (shape is None or own == shape) and t.is_contiguous():
        return own[1]
    if t.get_device() != device:
        raise ValueError(f"{what}: a tensor on GPU {device} expected, got one on {t.device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what}: {' or '.join(str(d) for d in dtypes)} expected, got {t.dtype}")
    if t.dim() != 2 or (shape is not None and t.shape != shape) or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: {'two dimensions' if shape is None else tuple(shape)} with contiguous rows expected, got "
                         f"{tuple(t.shape)} strides {t.stride()}")
    rows, cols = t.shape
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError(f"{what}: rows overlap (strides {t.stride()})")
    return ld


def _vector(t, n, dtypes, what, device, strided=False):
    """Check a 1-D tensor of n elements (contiguous, or any distance with ``strided``); the distance of its elements."""
    if t.get_device() == device and t.dtype in dtypes and t.dim() == 1 and t.numel() == n and t.is_contiguous():
        return 1
    if t.get_device() != device:
        raise ValueError(f"{what}: a tensor on GPU {device} expected, got one on {t.device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what}: {' or '.join(str(d) for d in dtypes)} expected, got {t.dtype}")
    if t.dim() != 1 or t.shape[0] != n or (not strided and n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: {n} {'' if strided else 'contiguous '}elements expected, got {tuple(t.shape)} strides {t.stride()}")
    return t.stride(0) if n > 1 else 1


def _address(t):
    return None if t is None else t.data_ptr()


_F32, _U8, _INT32 = (torch.float32,), (torch.uint8,), (torch.int32,)
_WITH_F32 = {torch.bfloat16: (torch.bfloat16, torch.float32), torch.float16: (torch.float16, torch.float32), torch.float32: _F32}

MATMUL_FWD, MATMUL_DGRAD, MATMUL_WGRAD = 0, 1, 2


def matmul_items(matmuls):
    """A ctypes array of ``fp8_matmul_item_t`` from (kind, a8, d_ba, b8, d_bb, out[, bias_vec[, d_amax_out]]) tuples
    (row-major operands: FWD x8, w8 -> y; DGRAD dy8, w8 -> dx; WGRAD dy8, x8 -> dw); build it once and hand it to
    ``Context.linear_group`` every step (the tensors must stay alive)."""
    arr = (MatmulItem * len(matmuls))()
    for it, m in zip(arr, matmuls):
        kind, a8, d_ba, b8, d_bb, out = m[:6]
        bias_vec = m[6] if len(m) > 6 else None
        d_amax_out = m[7] if len(m) > 7 else None
        if kind == MATMUL_FWD:
            (T, K), N = a8.shape, b8.shape[0]
        elif kind == MATMUL_DGRAD:
            (T, N), K = a8.shape, b8.shape[1]
        else:
            (T, N), K = a8.shape, b8.shape[1]
        it.kind, it.T, it.K, it.N = kind, T, K, N
        it.a8, it.d_ba, it.b8, it.d_bb = a8.data_ptr(), d_ba.data_ptr(), b8.data_ptr(), d_bb.data_ptr()
        it.bias_vec = bias_vec.data_ptr() if bias_vec is not None else None
        it.bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        it.out, it.out_dt = out.data_ptr(), _DT[out.dtype]
        it.d_amax_out = d_amax_out.data_ptr() if d_amax_out is not None else None
    return arr


# -- element-wise kernels of the stress stack (include/fp8_harness.h): harness, not the paper's method -----------------
def _bf16(t):
    assert t.dtype == torch.bfloat16 and t.is_contiguous() and t.is_cuda, "contiguous bf16 CUDA tensor expected"
    return t


def harness_gelu(x, y):
    _check(_lib.fp8h_gelu(_ptr(_bf16(x)), _ptr(_bf16(y)), x.numel(), _stream()), "fp8h_gelu")


def harness_gelu_backward(g, pre, out):
    _check(_lib.fp8h_gelu_backward(_ptr(_bf16(g)), _ptr(_bf16(pre)), _ptr(_bf16(out)), g.numel(), _stream()), "fp8h_gelu_backward")


def harness_mse_grad(y, target, scale, g):
    _check(_lib.fp8h_mse_grad(_ptr(_bf16(y)), _ptr(_bf16(target)), float(scale), _ptr(_bf16(g)), y.numel(), _stream()),
           "fp8h_mse_grad")


def harness_sgd(w32, dw, lr, w16):
    assert w32.dtype == torch.float32 and w32.is_contiguous()
    _check(_lib.fp8h_sgd(_ptr(w32), _ptr(_bf16(dw)), float(lr), _ptr(_bf16(w16)), w32.numel(), _stream()), "fp8h_sgd")


class Context:
    """Owns one ``fp8_ctx``.  All methods launch on torch's current stream."""

    def __init__(self, device: int = 0):
        self._h = c_void_p()
        self.device = device
        _check(_lib.fp8_create(byref(self._h), device), "fp8_create")

    def close(self):
        if self._h:
            _lib.fp8_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- status ---------------------------------------------------------------
    def device_flags(self, clear: bool = True) -> int:
        flags = c_uint(0)
        st = _lib.fp8_device_flags(self._h, _stream(), byref(flags), 1 if clear else 0)
        if st not in (OK, ERR_DEVICE_TIMEOUT):
            _check(st, "fp8_device_flags")
        return flags.value

    def selftest_wait_expiry(self, limit_ns: int = 1_000_000):
        """Make one bounded device-side wait run out on purpose (raises FP8_FLAG_TIMEOUT, no fault)."""
        _check(_lib.fp8_selftest_wait_expiry(self._h, ctypes.c_uint64(limit_ns), _stream()), "fp8_selftest_wait_expiry")

    def selftest_mma_ceiling(self, out, d_zero, K: int):
        """The CTA-pair matmul kernel on an out.shape[0] x out.shape[1] x K problem with its operand loads off."""
        _check(_lib.fp8_selftest_mma_ceiling(self._h, _ptr(out), _ptr(d_zero), out.shape[0], out.shape[1], K, _stream()),
               "fp8_selftest_mma_ceiling")

    # -- amax / bias ------------------------------------------------------------
    def amax(self, x, d_amax, rows=None, cols=None, ld=None):
        rows = x.shape[0] if rows is None else rows
        cols = x.shape[1] if cols is None else cols
        ld = _ld(x) if ld is None else ld
        _check(_lib.fp8_amax(self._h, _ptr(x), _DT[x.dtype], rows, cols, ld, _ptr(d_amax), _stream()), "fp8_amax")

    def scaling_bias(self, d_amax, fmt, conv, margin, d_bias):
        _check(_lib.fp8_scaling_bias(self._h, _ptr(d_amax), fmt, conv, margin, _ptr(d_bias), _stream()),
               "fp8_scaling_bias")

    def amax_history_bias(self, d_history, d_cursor, d_amax_new, fmt, d_bias, conv=CONV_PAPER, margin=0):
        _check(_lib.fp8_amax_history_bias(self._h, _ptr(d_history), d_history.numel(), _ptr(d_cursor), _ptr(d_amax_new),
                                          fmt, conv, margin, _ptr(d_bias), _stream()), "fp8_amax_history_bias")

    # -- bias log ---------------------------------------------------------------
    def bias_log_append(self, d_ring, d_head, step, first_tensor_id, d_amax, d_bias):
        """``fp8_bias_log_append``: d_ring is an int32 tensor [capacity, 4] (one ``fp8_bias_record_t`` per row: step,
        tensor id, amax bits, bias), d_head an int64 scalar tensor; d_amax / d_bias are 1-D device arrays."""
        _check(_lib.fp8_bias_log_append(self._h, _ptr(d_ring), d_ring.shape[0], _ptr(d_head), step, first_tensor_id,
                                        _ptr(d_amax), _ptr(d_bias), d_amax.numel(), _stream()), "fp8_bias_log_append")

    def bias_mode(self, d_ring, d_head, tensor_id, step_lo, step_hi, d_mode, d_count, d_samples=None):
        _check(_lib.fp8_bias_mode(self._h, _ptr(d_ring), d_ring.shape[0], _ptr(d_head), tensor_id, step_lo, step_hi,
                                  _ptr(d_mode), _ptr(d_count), _ptr(d_samples), _stream()), "fp8_bias_mode")

    # -- cast -------------------------------------------------------------------
    def _cast(self, fn, name, x, d_bias, conv, margin, d_amax_out, d_bias_out, y, y_t, rows, cols, ld):
        rows = x.shape[0] if rows is None else rows
        cols = x.shape[1] if cols is None else cols
        ld = _ld(x) if ld is None else ld
        _check(fn(self._h, _ptr(x), _DT[x.dtype], rows, cols, ld, _ptr(d_bias), conv, margin, _ptr(d_amax_out),
                  _ptr(d_bias_out), _ptr(y), _ptr(y_t), _stream()), name)

    def cast_e4(self, x, d_bias, conv=CONV_PAPER, margin=0, d_amax_out=None, d_bias_out=None, y=None, y_t=None,
                rows=None, cols=None, ld=None):
        self._cast(_lib.fp8_cast_e4, "fp8_cast_e4", x, d_bias, conv, margin, d_amax_out, d_bias_out, y, y_t, rows,
                   cols, ld)

    def cast_e5(self, x, d_bias, conv=CONV_PAPER, margin=0, d_amax_out=None, d_bias_out=None, y=None, y_t=None,
                rows=None, cols=None, ld=None):
        self._cast(_lib.fp8_cast_e5, "fp8_cast_e5", x, d_bias, conv, margin, d_amax_out, d_bias_out, y, y_t, rows,
                   cols, ld)

    def cast_predicted(self, fmt, x, d_amax_out, d_bias_inout, y, conv=CONV_PAPER, margin=0, rows=None, cols=None,
                       ld=None):
        rows = x.shape[0] if rows is None else rows
        cols = x.shape[1] if cols is None else cols
        ld = _ld(x) if ld is None else ld
        _check(_lib.fp8_cast_predicted(self._h, fmt, _ptr(x), _DT[x.dtype], rows, cols, ld, conv, margin,
                                       _ptr(d_amax_out), _ptr(d_bias_inout), _ptr(y), _stream()), "fp8_cast_predicted")

    def cast_group(self, items, conv=CONV_PAPER, predicted=False, mode=None):
        """``fp8_cast_group``.  `items`: a ``group_items(...)`` array, or a list of (fmt, x, d_amax, d_bias, y[, margin])
        tuples that is marshalled on the spot.  `mode`: one of the GROUP_* constants (default: GROUP_PREDICTED if
        `predicted` else GROUP_AMAX_CAST)."""
        arr = items if isinstance(items, ctypes.Array) else group_items(items)
        if mode is None:
            mode = GROUP_PREDICTED if predicted else GROUP_AMAX_CAST
        _check(_lib.fp8_cast_group(self._h, arr, len(arr), conv, mode, _stream()), "fp8_cast_group")

    def prediction_stats(self, clear: bool = True):
        hits, misses = c_uint(0), c_uint(0)
        _check(_lib.fp8_prediction_stats(self._h, _stream(), byref(hits), byref(misses), 1 if clear else 0),
               "fp8_prediction_stats")
        return hits.value, misses.value

    def range_stats(self, fmt, x, d_bias, d_counts, conv=CONV_PAPER, rows=None, cols=None, ld=None):
        """d_counts: 4 x int64 on the device = clipped, flushed to zero, subnormal, non-zero finite."""
        rows = x.shape[0] if rows is None else rows
        cols = x.shape[1] if cols is None else cols
        ld = _ld(x) if ld is None else ld
        _check(_lib.fp8_range_stats(self._h, fmt, _ptr(x), _DT[x.dtype], rows, cols, ld, _ptr(d_bias), conv,
                                    _ptr(d_counts), _stream()), "fp8_range_stats")

    def ptq_weights(self, w, conv, w8, w8_t, d_bw, d_amax_w):
        _check(_lib.fp8_ptq_weights(self._h, _ptr(w), _DT[w.dtype], w.shape[0], w.shape[1], _ld(w), conv,
                                    _ptr(w8), _ptr(w8_t), _ptr(d_bw), _ptr(d_amax_w), _stream()), "fp8_ptq_weights")

    # -- matmuls ----------------------------------------------------------------
    def linear_fwd(self, x8, d_bx, w8, d_bw, y, bias_vec=None, d_amax_y=None, conv=CONV_PAPER):
        T, K = x8.shape
        N = w8.shape[0]
        bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        _check(_lib.fp8_linear_fwd(self._h, _ptr(x8), _ptr(d_bx), _ptr(w8), _ptr(d_bw), _ptr(bias_vec), bias_dt,
                                   _ptr(y), _DT[y.dtype], _ptr(d_amax_y), T, K, N, conv, _stream()),
               "fp8_linear_fwd")

    def linear_infer(self, x8, d_bx, w8, d_bw, y, bias_vec=None, d_amax_y=None, conv=CONV_PAPER):
        """``fp8_linear_infer``: linear_fwd for weights whose bytes were final before the launch ahead of this call."""
        T, K = x8.shape
        N = w8.shape[0]
        bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        _check(_lib.fp8_linear_infer(self._h, _ptr(x8), _ptr(d_bx), _ptr(w8), _ptr(d_bw), _ptr(bias_vec), bias_dt,
                                     _ptr(y), _DT[y.dtype], _ptr(d_amax_y), T, K, N, conv, _stream()),
               "fp8_linear_infer")

    def linear_infer_cast(self, x, d_amax_x, d_bx, x8, w8, d_bw, y, margin=0, bias_vec=None, d_amax_y=None, conv=CONV_PAPER):
        """``fp8_linear_infer_cast``: FP8-AMAX of the activation x and the forward matmul on weights quantised once."""
        T, K = x.shape
        N = w8.shape[0]
        bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        _check(_lib.fp8_linear_infer_cast(self._h, _ptr(x), _DT[x.dtype], margin, _ptr(d_amax_x), _ptr(d_bx), _ptr(x8),
                                          _ptr(w8), _ptr(d_bw), _ptr(bias_vec), bias_dt, _ptr(y), _DT[y.dtype],
                                          _ptr(d_amax_y), T, K, N, conv, _stream()), "fp8_linear_infer_cast")

    def linear_group(self, items, conv=CONV_PAPER):
        """``fp8_linear_group``: independent matmuls in one launch.  `items`: a ``matmul_items(...)`` array or the list
        of tuples it is built from."""
        arr = items if isinstance(items, ctypes.Array) else matmul_items(items)
        _check(_lib.fp8_linear_group(self._h, arr, len(arr), conv, _stream()), "fp8_linear_group")

    def linear_fwd_act(self, x8, d_bx, w8, d_bw, y_pre, y_act, bias_vec=None, d_amax_act=None, act=ACT_GELU,
                       conv=CONV_PAPER):
        T, K = x8.shape
        N = w8.shape[0]
        bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        _check(_lib.fp8_linear_fwd_act(self._h, _ptr(x8), _ptr(d_bx), _ptr(w8), _ptr(d_bw), _ptr(bias_vec), bias_dt,
                                       _ptr(y_pre), _ptr(y_act), act, _ptr(d_amax_act), T, K, N, conv, _stream()),
               "fp8_linear_fwd_act")

    def linear_dgrad(self, dy8, d_bg, w8, w8_t, d_bw, dx, d_amax_dx=None, conv=CONV_PAPER):
        T, N = dy8.shape
        K = dx.shape[1]
        _check(_lib.fp8_linear_dgrad(self._h, _ptr(dy8), _ptr(d_bg), _ptr(w8), _ptr(w8_t), _ptr(d_bw), _ptr(dx),
                                     _DT[dx.dtype], _ptr(d_amax_dx), T, K, N, conv, _stream()), "fp8_linear_dgrad")

    def linear_dgrad_act(self, dy8, d_bg, w8, w8_t, d_bw, y_pre, dx, dx_act, d_amax_act=None, act=ACT_GELU,
                         conv=CONV_PAPER):
        T, N = dy8.shape
        K = w8.shape[1] if w8 is not None else w8_t.shape[0]
        _check(_lib.fp8_linear_dgrad_act(self._h, _ptr(dy8), _ptr(d_bg), _ptr(w8), _ptr(w8_t), _ptr(d_bw), _ptr(y_pre),
                                         _ptr(dx), _ptr(dx_act), act, _ptr(d_amax_act), T, K, N, conv, _stream()),
               "fp8_linear_dgrad_act")

    def linear_fwd_q(self, x8, d_bx, w8, d_bw, z8, d_bz, y_pre=None, z=None, bias_vec=None, d_amax_z=None,
                     act=ACT_NONE, conv=CONV_PAPER):
        T, K = x8.shape
        N = w8.shape[0]
        bias_dt = _DT[bias_vec.dtype] if bias_vec is not None else BF16
        _check(_lib.fp8_linear_fwd_q(self._h, _ptr(x8), _ptr(d_bx), _ptr(w8), _ptr(d_bw), _ptr(bias_vec), bias_dt, act,
                                     _ptr(y_pre), _ptr(z), _ptr(z8), _ptr(d_bz), _ptr(d_amax_z), T, K, N, conv,
                                     _stream()), "fp8_linear_fwd_q")

    def linear_dgrad_q(self, dy8, d_bg, w8, w8_t, d_bw, g8, d_bq, y_pre=None, dx=None, g=None, d_amax_g=None,
                       act=ACT_NONE, conv=CONV_PAPER):
        T, N = dy8.shape
        K = w8.shape[1] if w8 is not None else w8_t.shape[0]
        _check(_lib.fp8_linear_dgrad_q(self._h, _ptr(dy8), _ptr(d_bg), _ptr(w8), _ptr(w8_t), _ptr(d_bw), act,
                                       _ptr(y_pre), _ptr(dx), _ptr(g), _ptr(g8), _ptr(d_bq), _ptr(d_amax_g), T, K, N,
                                       conv, _stream()), "fp8_linear_dgrad_q")

    def linear_f16acc(self, kind, a8, d_ba, b8, d_bb, out, T, K, N, chunk=128, conv=CONV_PAPER):
        """``fp8_linear_f16acc``: the matmul of `kind` with FP16 accumulation emulated; out is float16 or float32."""
        _check(_lib.fp8_linear_f16acc(self._h, kind, _ptr(a8), _ptr(d_ba), _ptr(b8), _ptr(d_bb), _ptr(out), _DT[out.dtype],
                                      chunk, T, K, N, conv, _stream()), "fp8_linear_f16acc")

    def linear_wgrad(self, dy8, dy8_t, d_bg, x8, x8_t, d_bx, dw, T, conv=CONV_PAPER):
        N, K = dw.shape
        _check(_lib.fp8_linear_wgrad(self._h, _ptr(dy8), _ptr(dy8_t), _ptr(d_bg), _ptr(x8), _ptr(x8_t), _ptr(d_bx),
                                     _ptr(dw), _DT[dw.dtype], T, K, N, conv, _stream()), "fp8_linear_wgrad")

    # -- paged FP8 cache (calls without rows check their arguments and launch nothing) -------------
    def _kv(self, fn, name, cache, batch, k, v):
        some = k if k is not None else v
        if some is None:
            raise ValueError("keys, values or both")
        heads, dim = cache.kv_heads, cache.head_dim
        _check_handles(cache, batch, self.device)
        ld_k = _rows3(k, heads, dim, "keys", self.device) if k is not None else 0
        ld_v = _rows3(v, heads, dim, "values", self.device) if v is not None else 0
        if k is not None and v is not None and (k.dtype != v.dtype or k.shape[0] != v.shape[0]):
            raise ValueError("keys and values of one shape and type")
        dt = _DT.get(some.dtype)
        if dt is None:
            raise ValueError(f"keys and values: bf16, fp16 or fp32, got {some.dtype}")
        if some.shape[0] == 0:
            return
        status = fn(self._h, cache._ref, batch._of(some.shape[0]), None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                    dt, ld_k, ld_v, cache.conv, _raw_stream(self.device))
        if status:
            _check(status, name)

    def kv_append(self, cache, batch, k, v):
        """``fp8_kv_append``: quantise the new tokens' keys and values, [tokens, kv_heads, head_dim], into the cache."""
        self._kv(_lib.fp8_kv_append, "fp8_kv_append", cache, batch, k, v)

    def kv_read(self, cache, batch, k, v):
        """``fp8_kv_read``: the numbers that the cache holds, into k and v (either may be None)."""
        self._kv(_lib.fp8_kv_read, "fp8_kv_read", cache, batch, k, v)

    def attn_paged(self, cache, batch, q, out, scale=None, causal=True, lse=None):
        """``fp8_attn_paged``: q, out [tokens, q_heads, head_dim] bf16, lse float32 [tokens, q_heads] or None; scale
        1 / sqrt(head_dim) by default."""
        shape, dim = q.shape, cache.head_dim
        if len(shape) != 3:
            raise ValueError(f"q: [tokens, q_heads, {dim}] expected, got {tuple(shape)}")
        heads = shape[1]
        _check_handles(cache, batch, self.device)
        ld_q, ld_o = _rows3(q, heads, dim, "q", self.device), _rows3(out, heads, dim, "out", self.device)
        if q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16 or out.shape[0] != shape[0]:
            raise ValueError("q and out: bf16 tensors of one shape")
        lse_ptr = None
        if lse is not None:
            if lse.dtype != torch.float32 or lse.shape != shape[:2] or not lse.is_contiguous() or lse.get_device() != self.device:
                raise ValueError("lse: contiguous float32 [tokens, q_heads] on the context's GPU")
            lse_ptr = lse.data_ptr()
        if shape[0] == 0:
            return
        status = _lib.fp8_attn_paged(self._h, cache._ref, batch._of(shape[0]), q.data_ptr(), ld_q, heads, out.data_ptr(), ld_o, lse_ptr,
                                     dim ** -0.5 if scale is None else scale, 1 if causal else 0, cache.conv,
                                     _raw_stream(self.device))
        if status:
            _check(status, "fp8_attn_paged")

    # -- norm between two linears (include/fp8_norm.h); calls without rows check their arguments and launch nothing -------
    def norm_fwd(self, x, weight=None, bias_vec=None, residual=None, eps=1e-5, kind=NORM_LAYER, h=None, y=None, d_mean=None,
                 d_rstd=None, y8=None, d_bias=None, d_amax_out=None, d_bias_out=None, conv=CONV_PAPER, margin=0):
        """``fp8_norm_fwd``: x, residual, h, y [rows, cols] of one type; weight, bias_vec [cols] of that type or float32;
        y8 uint8 [rows, cols]; d_bias: the bias to cast under, None for that of Eq. 3 (d_bias_out)."""
        dev, dtype = self.device, x.dtype
        ld_x = _matrix(x, None, _DT, "x", dev)
        shape, dt = x.shape, (dtype,)
        rows, cols = shape
        ld_r = ld_h = ld_y = p_r = p_h = p_y = p_y8 = p_mean = p_rstd = p_b = p_a = p_o = 0
        if residual is not None:
            ld_r, p_r = _matrix(residual, shape, dt, "residual", dev), residual.data_ptr()
        if h is not None:
            ld_h, p_h = _matrix(h, shape, dt, "h", dev), h.data_ptr()
        if y is not None:
            ld_y, p_y = _matrix(y, shape, dt, "y", dev), y.data_ptr()
        if y8 is not None:
            if _matrix(y8, shape, _U8, "y8", dev) != cols:
                raise ValueError("y8: contiguous bytes expected")
            p_y8 = y8.data_ptr()
        w_dt, p_w = self._coefficients(weight, cols, dtype, None, "weight")
        w_dt, p_v = self._coefficients(bias_vec, cols, dtype, w_dt, "bias_vec")
        if d_mean is not None:
            _vector(d_mean, rows, _F32, "d_mean", dev)
            p_mean = d_mean.data_ptr()
        if d_rstd is not None:
            _vector(d_rstd, rows, _F32, "d_rstd", dev)
            p_rstd = d_rstd.data_ptr()
        if d_bias is not None:
            _vector(d_bias, 1, _INT32, "d_bias", dev)
            p_b = d_bias.data_ptr()
        if d_amax_out is not None:
            _vector(d_amax_out, 1, _F32, "d_amax_out", dev)
            p_a = d_amax_out.data_ptr()
        if d_bias_out is not None:
            _vector(d_bias_out, 1, _INT32, "d_bias_out", dev)
            p_o = d_bias_out.data_ptr()
        if rows == 0:
            return
        code = _DT[dtype]
        status = _lib.fp8_norm_fwd(self._h, _NORM_FWD.pack(x.data_ptr(), p_r, p_w, p_v, p_h, p_y, p_mean, p_rstd, p_y8, p_b, p_a, p_o, rows,
                                                           cols, ld_x, ld_r, ld_h, ld_y, kind, code, code if w_dt is None else _DT[w_dt],
                                                           conv, margin, eps), _raw_stream(dev))
        if status:
            _check(status, "fp8_norm_fwd")

    def norm_bwd(self, dy, h, weight, d_mean, d_rstd, dx, dh=None, dw=None, db=None, d_amax=None, kind=NORM_LAYER):
        """``fp8_norm_bwd``: dy, h, dh, dx [rows, cols] of one type; weight, dw, db [cols] of that type or float32; d_mean
        (None for NORM_RMS), d_rstd float32 [rows]."""
        dev, dtype = self.device, dy.dtype
        ld_dy = _matrix(dy, None, _DT, "dy", dev)
        shape, dt = dy.shape, (dtype,)
        rows, cols = shape
        ld_dh = ld_dx = p_dh = p_dx = p_mean = p_rstd = p_a = 0
        ld_h = _matrix(h, shape, dt, "h", dev)
        if dh is not None:
            ld_dh, p_dh = _matrix(dh, shape, dt, "dh", dev), dh.data_ptr()
        if dx is not None:
            ld_dx, p_dx = _matrix(dx, shape, dt, "dx", dev), dx.data_ptr()
        w_dt, p_w = self._coefficients(weight, cols, dtype, None, "weight")
        w_dt, p_dw = self._coefficients(dw, cols, dtype, w_dt, "dw")
        w_dt, p_db = self._coefficients(db, cols, dtype, w_dt, "db")
        if d_mean is not None:
            _vector(d_mean, rows, _F32, "d_mean", dev)
            p_mean = d_mean.data_ptr()
        if d_rstd is not None:
            _vector(d_rstd, rows, _F32, "d_rstd", dev)
            p_rstd = d_rstd.data_ptr()
        if d_amax is not None:
            _vector(d_amax, 1, _F32, "d_amax", dev)
            p_a = d_amax.data_ptr()
        if rows == 0:
            for t in (dw, db):
                if t is not None:
                    t.zero_()
            return
        code = _DT[dtype]
        status = _lib.fp8_norm_bwd(self._h, _NORM_BWD.pack(dy.data_ptr(), h.data_ptr(), p_dh, p_w, p_mean, p_rstd, p_dx, p_dw, p_db, p_a, rows,
                                                           cols, ld_dy, ld_h, ld_dh, ld_dx, kind, code, code if w_dt is None else _DT[w_dt],
                                                           0), _raw_stream(dev))
        if status:
            _check(status, "fp8_norm_bwd")

    def _coefficients(self, t, cols, dtype, others, what):
        """Check a vector of ``cols`` elements of ``dtype`` or float32, all of a call's of one type (``others``, None: the
        first); that type and the address."""
        if t is None:
            return others, 0
        own = t.dtype
        _vector(t, cols, _WITH_F32[dtype], what, self.device)
        if others is not None and own != others:
            raise ValueError(f"{what}: the type of the other vectors ({others}) expected, got {own}")
        return own, t.data_ptr()

    # -- a head's losses (include/fp8_loss.h); calls without rows check their arguments and launch nothing -----------------
    def _logits(self, logits, scale):
        ld = _matrix(logits, None, _DT, "logits", self.device)
        rows, vocab = logits.shape
        return rows, (self._h, logits.data_ptr(), _DT[logits.dtype], ld, rows, vocab, scale)

    def _saved(self, saved, rows):
        if saved is not None and _matrix(saved, (rows, LOSS_SAVED), _F32, "saved", self.device) != LOSS_SAVED:
            raise ValueError("saved: contiguous float32 [rows, 4] expected")
        return _address(saved)

    def _row_numbers(self, t, rows, what):
        """Pointer and stride of one float32 a row (None: no pointer)."""
        if t is None:
            return None, 0
        return t.data_ptr(), _vector(t, rows, _F32, what, self.device, strided=True)

    def token_logprobs(self, logits, targets=None, scale=1.0, logprob=None, entropy=None, lse=None, saved=None, top_logprob=None,
                       top_index=None):
        """``fp8_token_logprobs``: logits [rows, vocab] bf16, fp16 or fp32; targets int32 or int64 [rows] (negative: none);
        logprob, entropy, lse float32 [rows]; saved float32 [rows, 4]; top_logprob float32 and top_index (the type of
        targets) [rows, k]."""
        rows, args = self._logits(logits, scale)
        for t, what in ((logprob, "logprob"), (entropy, "entropy"), (lse, "lse")):
            if t is not None:
                _vector(t, rows, _F32, what, self.device)
        it = targets.dtype if targets is not None else top_index.dtype if top_index is not None else torch.int32
        if targets is not None:
            _vector(targets, rows, _IT, "targets", self.device)
        k = 0
        if (top_logprob is None) != (top_index is None):
            raise ValueError("top_logprob and top_index go together")
        if top_index is not None:
            k = top_index.shape[-1]
            for t, want, what in ((top_index, (it,) if targets is not None else _IT, "top_index"), (top_logprob, _F32, "top_logprob")):
                if _matrix(t, (rows, k), want, what, self.device) != k:
                    raise ValueError(f"{what}: contiguous [rows, k] expected")
        keep = self._saved(saved, rows)
        if rows == 0:
            return
        status = _lib.fp8_token_logprobs(*args, _address(targets), _IT[it], _address(logprob), _address(entropy), _address(lse), keep, k,
                                         _address(top_logprob), _address(top_index), _raw_stream(self.device))
        if status:
            _check(status, "fp8_token_logprobs")

    def token_logprobs_bwd(self, logits, targets, saved, dlogits, g_logprob=None, g_entropy=None, scale=1.0, d_amax=None):
        """``fp8_token_logprobs_bwd``: saved as the forward call left it; g_logprob, g_entropy float32 [rows], any stride;
        dlogits like logits (or logits itself)."""
        rows, args = self._logits(logits, scale)
        ld_d = _matrix(dlogits, logits.shape, (logits.dtype,), "dlogits", self.device)
        if targets is not None:
            _vector(targets, rows, _IT, "targets", self.device)
        if d_amax is not None:
            _vector(d_amax, 1, _F32, "d_amax", self.device)
        keep = self._saved(saved, rows)
        g_lp, g_h = self._row_numbers(g_logprob, rows, "g_logprob"), self._row_numbers(g_entropy, rows, "g_entropy")
        if rows == 0:
            return
        status = _lib.fp8_token_logprobs_bwd(*args, _address(targets), I32 if targets is None else _IT[targets.dtype], keep, *g_lp, *g_h,
                                             dlogits.data_ptr(), ld_d, _address(d_amax), _raw_stream(self.device))
        if status:
            _check(status, "fp8_token_logprobs_bwd")

    def _teacher(self, index, value, rows, rest):
        if index.dim() != 2 or index.shape[0] != rows:
            raise ValueError(f"index: [{rows}, listed] expected, got {tuple(index.shape)}")
        ld_i = _matrix(index, index.shape, _IT, "index", self.device)
        ld_v = _matrix(value, index.shape, _F32, "value", self.device)
        return index.data_ptr(), _IT[index.dtype], ld_i, value.data_ptr(), ld_v, index.shape[1], DISTILL_REST if rest else DISTILL_TOP

    def distill_fwd(self, logits, index, value, loss, rest=True, scale=1.0, saved=None):
        """``fp8_distill_fwd``: index int32 or int64, value float32 [rows, listed] (what ``token_logprobs`` writes as
        top_index and top_logprob); loss float32 [rows]; saved float32 [rows, 4]."""
        rows, args = self._logits(logits, scale)
        teacher = self._teacher(index, value, rows, rest)
        _vector(loss, rows, _F32, "loss", self.device)
        keep = self._saved(saved, rows)
        if rows == 0:
            return
        status = _lib.fp8_distill_fwd(*args, *teacher, loss.data_ptr(), keep, _raw_stream(self.device))
        if status:
            _check(status, "fp8_distill_fwd")

    def distill_bwd(self, logits, index, value, saved, g_loss, dlogits, rest=True, scale=1.0, d_amax=None):
        """``fp8_distill_bwd``: saved as the forward call left it; g_loss float32 [rows], any stride; dlogits like logits (or
        logits itself)."""
        rows, args = self._logits(logits, scale)
        teacher = self._teacher(index, value, rows, rest)
        ld_d = _matrix(dlogits, logits.shape, (logits.dtype,), "dlogits", self.device)
        if d_amax is not None:
            _vector(d_amax, 1, _F32, "d_amax", self.device)
        keep, g = self._saved(saved, rows), self._row_numbers(g_loss, rows, "g_loss")
        if rows == 0:
            return
        status = _lib.fp8_distill_bwd(*args, *teacher, keep, *g, dlogits.data_ptr(), ld_d, _address(d_amax), _raw_stream(self.device))
        if status:
            _check(status, "fp8_distill_bwd")


def raw():
    """The ctypes library handle (for tests of the C ABI itself)."""
    return _lib
