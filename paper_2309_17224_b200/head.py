"""The head of a language model: its final norm and FP8 vocabulary matmul, and what is computed from the logits
(``include/fp8_loss.h``), wired into autograd.

``token_logprobs``   log probabilities of given tokens and the entropies of their rows (scoring, fine-tuning)
``top_tokens``       the most probable tokens and their log probabilities
``distill_loss``     divergence from a teacher's most probable tokens, as ``top_tokens`` lists them at the same ``scale``
``Fp8Head``          norm -> FP8 linear -> any of these

Logits are bf16, fp16 or fp32, [..., columns].  ``vocab``: how many of the columns are tokens (all of them by default; the
matmul's rows come in whole sixteens); the others are not looked at and have no gradient.  ``scale`` is 1 / temperature.
Everything numeric happens in the library.
"""
from __future__ import annotations

from typing import Optional

import torch

from .module import Fp8NormLinear, default_context, matrix_rows


def _tokens(logits, vocab):
    """The logits' token columns as [rows, vocab]."""
    columns = logits.shape[-1]
    vocab = columns if vocab is None else vocab
    if not 0 < vocab <= columns:
        raise ValueError(f"vocab 1 .. {columns} expected, got {vocab}")
    return matrix_rows(logits, columns)[:, :vocab]


def _gradient(logits, vocab):
    """A gradient of the logits and its token columns, the others zero."""
    columns = logits.shape[-1]
    full = torch.empty((logits.numel() // columns, columns), dtype=logits.dtype, device=logits.device)
    if vocab < columns:
        full[:, vocab:].zero_()
    return full, full[:, :vocab]


def _context(logits, ctx):
    return ctx if ctx is not None else default_context(logits.get_device())


class _TokenLogprobsFn(torch.autograd.Function):
    @staticmethod
    def forward(fn, logits, targets, vocab, scale, lib):
        x = _tokens(logits, vocab)
        rows = x.shape[0]
        f32 = dict(dtype=torch.float32, device=x.device)
        logprob, entropy, saved = torch.empty(rows, **f32), torch.empty(rows, **f32), torch.empty((rows, 4), **f32)
        flat = targets.reshape(-1).contiguous()
        lib.token_logprobs(x, flat, scale=scale, logprob=logprob, entropy=entropy, saved=saved)
        fn.lib, fn.scale, fn.vocab = lib, scale, x.shape[1]
        fn.set_materialize_grads(False)
        fn.save_for_backward(logits, flat, saved)
        return logprob.reshape(targets.shape), entropy.reshape(targets.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, g_logprob, g_entropy):
        if g_logprob is None and g_entropy is None:
            return None, None, None, None, None
        logits, targets, saved = fn.saved_tensors
        full, part = _gradient(logits, fn.vocab)
        fn.lib.token_logprobs_bwd(_tokens(logits, fn.vocab), targets, saved, part, scale=fn.scale,
                                  g_logprob=None if g_logprob is None else g_logprob.reshape(-1),
                                  g_entropy=None if g_entropy is None else g_entropy.reshape(-1))
        return full.reshape(logits.shape), None, None, None, None


class _DistillFn(torch.autograd.Function):
    @staticmethod
    def forward(fn, logits, index, value, vocab, scale, rest, lib):
        x = _tokens(logits, vocab)
        rows, listed = x.shape[0], index.shape[-1]
        loss = torch.empty(rows, dtype=torch.float32, device=x.device)
        saved = torch.empty((rows, 4), dtype=torch.float32, device=x.device)
        index, value = index.reshape(-1, listed).contiguous(), value.reshape(-1, listed).contiguous()
        lib.distill_fwd(x, index, value, loss, rest=rest, scale=scale, saved=saved)
        fn.lib, fn.scale, fn.rest, fn.vocab = lib, scale, rest, x.shape[1]
        fn.save_for_backward(logits, index, value, saved)
        return loss.reshape(logits.shape[:-1])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(fn, g_loss):
        logits, index, value, saved = fn.saved_tensors
        full, part = _gradient(logits, fn.vocab)
        fn.lib.distill_bwd(_tokens(logits, fn.vocab), index, value, saved, g_loss.reshape(-1), part, rest=fn.rest, scale=fn.scale)
        return full.reshape(logits.shape), None, None, None, None, None, None


def token_logprobs(logits, targets, scale: float = 1.0, vocab: Optional[int] = None, ctx=None):
    """(log probabilities of the given tokens, entropies), float32 of targets' shape (int32 or int64, one per row of logits).  A
    negative target: none is given, 0 and no gradient.  Cross entropy is the first one's negative."""
    if targets.shape != logits.shape[:-1]:
        raise ValueError(f"targets {tuple(logits.shape[:-1])} expected, got {tuple(targets.shape)}")
    return _TokenLogprobsFn.apply(logits, targets, vocab, scale, _context(logits, ctx))


@torch.no_grad()
def top_tokens(logits, k: int, scale: float = 1.0, vocab: Optional[int] = None, ctx=None):
    """(log probabilities float32, tokens int64), [..., k], by falling probability, equal ones by rising token number."""
    x = _tokens(logits, vocab)
    value = torch.empty((x.shape[0], k), dtype=torch.float32, device=x.device)
    index = torch.empty((x.shape[0], k), dtype=torch.int64, device=x.device)
    _context(logits, ctx).token_logprobs(x, scale=scale, top_logprob=value, top_index=index)
    shape = (*logits.shape[:-1], k)
    return value.reshape(shape), index.reshape(shape)


def distill_loss(logits, index, value, scale: float = 1.0, rest: bool = True, vocab: Optional[int] = None, ctx=None):
    """Divergence of the student's logits from the teacher's lists, float32, one a row: index (int32 or int64, negative:
    padding) and value (float32 log probabilities), [..., listed].  ``rest``: all other tokens are one more outcome with what
    the list leaves; otherwise the listed ones share everything.  The lists are the teacher's: no gradient reaches them."""
    if index.shape[:-1] != logits.shape[:-1] or value.shape != index.shape:
        raise ValueError(f"index and value {tuple(logits.shape[:-1])} + (listed,) expected, got {tuple(index.shape)}, {tuple(value.shape)}")
    return _DistillFn.apply(logits, index, value, vocab, scale, rest, _context(logits, ctx))


class Fp8Head(Fp8NormLinear):
    """Final norm and vocabulary matmul in FP8; ``forward`` gives the logits of whole sixteens of columns, of which the first
    ``vocab`` are tokens, the methods what is computed from them."""

    def __init__(self, hidden: int, vocab: int, **kw):
        super().__init__(hidden, -(-vocab // 16) * 16, **kw)
        self.vocab = vocab

    def _logits(self, x, residual):
        y = self(x, residual)
        return y if residual is None else y[0]

    def logprobs(self, x, targets, residual=None, scale: float = 1.0):
        return token_logprobs(self._logits(x, residual), targets, scale, self.vocab, self.ctx)

    @torch.no_grad()
    def top(self, x, k: int, residual=None, scale: float = 1.0):
        return top_tokens(self._logits(x, residual), k, scale, self.vocab, self.ctx)

    def distill(self, x, index, value, residual=None, scale: float = 1.0, rest: bool = True):
        return distill_loss(self._logits(x, residual), index, value, scale, rest, self.vocab, self.ctx)
