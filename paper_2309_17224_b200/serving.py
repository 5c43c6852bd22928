"""Inference with an FP8 key/value cache: pages, and a self-attention layer between two FP8 linears.

What a serving program puts around the operators of ``include/fp8_kv.h``:

``PagePool``            which pages of the cache belong to which sequence (host bookkeeping, no device work except the three
                        small index tensors of a call).
``Fp8SelfAttention``    QKV linear -> ``fp8_kv_append`` -> ``fp8_attn_paged`` -> output linear, for chunks of a prompt and
                        for single tokens alike; the linears are ``module.Fp8Linear`` in ``eval()`` mode (weights quantised
                        once, Section 3.1 of the paper).

Everything numeric happens in the library.  A position encoding, if the model has one, is the caller's: ``rotate`` is
called with the query and key views of the QKV output before they are used.
"""
from __future__ import annotations

from typing import Callable, Dict, List, Optional, Sequence

import torch

from . import fp8lin
from .module import Fp8Linear, default_context


class PagePool:
    """Pages of one cache shape, handed out to sequences as they grow; layers share the numbering."""

    def __init__(self, pages: int, page_size: int):
        if pages <= 0 or page_size not in (16, 32, 64, 128):
            raise ValueError("pages > 0, page_size 16, 32, 64 or 128")
        self.page_size = page_size
        self._free: List[int] = list(range(pages - 1, -1, -1))
        self._pages: Dict[object, List[int]] = {}
        self._length: Dict[object, int] = {}

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq) -> int:
        """Tokens that the sequence holds (0 for one that is not known)."""
        return self._length.get(seq, 0)

    def extend(self, seqs: Sequence, new_tokens: Sequence[int]) -> None:
        """Make room for each sequence's new tokens; all of them or, if the pages do not suffice, none (MemoryError)."""
        if len(set(seqs)) != len(seqs) or len(seqs) != len(new_tokens) or any(n < 0 for n in new_tokens):
            raise ValueError("distinct sequences and a number of new tokens for each")
        size = self.page_size
        need = [-(-(self.length(s) + n) // size) - len(self._pages.get(s, ())) for s, n in zip(seqs, new_tokens)]
        if sum(need) > len(self._free):
            raise MemoryError(f"{sum(need)} pages needed, {len(self._free)} free")
        for s, n, k in zip(seqs, new_tokens, need):
            self._pages.setdefault(s, []).extend(self._free.pop() for _ in range(k))
            self._length[s] = self.length(s) + n

    def release(self, seq) -> None:
        """Give a sequence's pages back."""
        self._free.extend(reversed(self._pages.pop(seq, [])))
        self._length.pop(seq, None)

    def indices(self, seqs: Sequence, new_tokens: Sequence[int]):
        """(q_start, kv_len, page_table rows) as host lists, for sequences that ``extend`` has made room in."""
        start = [0]
        for n in new_tokens:
            start.append(start[-1] + n)
        lens = [self.length(s) for s in seqs]
        width = max([1] + [-(-n // self.page_size) for n in lens])
        rows = [(self._pages.get(s, []) + [0] * width)[:width] for s in seqs]
        return start, lens, rows

    def batch(self, seqs: Sequence, new_tokens: Sequence[int], device="cuda") -> "fp8lin.SeqBatch":
        """The index tensors of a step, for all layers of it: new storage and three copies from host memory that the caller
        waits for (48 us for one sequence of 64 pages, 104 for 16, 274 for 64).  A captured graph keeps reading the tensors that
        it was captured with: a program that replays one keeps a batch and copies new starts, lengths and pages into it."""
        start, lens, rows = self.indices(seqs, new_tokens)
        i32 = dict(dtype=torch.int32, device=device)
        return fp8lin.SeqBatch(torch.tensor(start, **i32), torch.tensor(lens, **i32),
                               torch.tensor(rows, **i32).view(len(lens), -1 if lens else 1),
                               max_q_len=max([1, *new_tokens]), max_kv_len=max([1, *lens]))


def empty_cache(pages: int, kv_heads: int, page_size: int, head_dim: int, conv: int = fp8lin.CONV_PAPER, device="cuda"):
    """The pages of one layer, uninitialised (what no token was written to is never read).  With CONV_PAPER, the convention of
    the linears, about one row in twenty clips its largest numbers by up to a fifteenth and raises FLAG_SATURATED; with
    CONV_NATIVE none does."""
    k8, v8 = (torch.empty((pages, kv_heads, page_size, head_dim), dtype=torch.uint8, device=device) for _ in range(2))
    bk, bv = (torch.empty((pages, kv_heads, page_size), dtype=torch.int8, device=device) for _ in range(2))
    return fp8lin.KvCache(k8, v8, bk, bv, conv=conv)


class Fp8SelfAttention(torch.nn.Module):
    """Self-attention of a decoder layer for inference: x [tokens, hidden] bf16, fp16 or fp32 -> [tokens, hidden] bf16.

    The tokens are those of ``batch`` (``PagePool.batch``), sequence after sequence; their keys and values enter ``cache``
    and each attends causally to its sequence's cached tokens.  Calls that share ``ctx`` (by default the device's
    ``default_context``) must not overlap on the GPU: a program that runs prefill and decoding on two streams gives the layers
    of each a context of its own."""

    def __init__(self, hidden: int, q_heads: int, kv_heads: int, head_dim: int, cache: "fp8lin.KvCache", device="cuda",
                 rotate: Optional[Callable[[torch.Tensor, torch.Tensor, "fp8lin.SeqBatch"], None]] = None,
                 ctx: Optional["fp8lin.Context"] = None):
        super().__init__()
        if q_heads % kv_heads or (cache.kv_heads, cache.head_dim) != (kv_heads, head_dim):
            raise ValueError("q_heads a multiple of kv_heads; the cache has this layer's kv_heads and head_dim")
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.cache, self.rotate = cache, rotate
        self.ctx = ctx if ctx is not None else default_context(torch.device(device).index or 0)
        # (attention reads bf16 queries whatever x is)
        self.qkv = Fp8Linear(hidden, (q_heads + 2 * kv_heads) * head_dim, device=device, out_dtype=torch.bfloat16, ctx=self.ctx)
        self.out = Fp8Linear(q_heads * head_dim, hidden, device=device, ctx=self.ctx)
        self.eval()

    @torch.no_grad()
    def forward(self, x: torch.Tensor, batch: "fp8lin.SeqBatch") -> torch.Tensor:
        if x.shape[0] == 0:                  # no sequence has new tokens
            return torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
        hq, hk = self.q_heads, self.kv_heads
        qkv = self.qkv(x).unflatten(1, (hq + 2 * hk, self.head_dim))
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        if self.rotate is not None:
            self.rotate(q, k, batch)
        self.ctx.kv_append(self.cache, batch, k, v)
        o = torch.empty((x.shape[0], hq, self.head_dim), dtype=torch.bfloat16, device=x.device)
        self.ctx.attn_paged(self.cache, batch, q, o, causal=True)
        return self.out(o.flatten(1))
