"""Plain 64-bit implementations of the cache operators, for the tests: numpy / torch on the CPU, row by row."""
import numpy as np
import torch

import oracle as O


def e4_table():
    """The 256 numbers of E4M3 (0x7F and 0xFF are NaN), from the format's definition."""
    t = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        t[c] = np.nan if (c & 127) == 127 else mag
        if c & 128:
            t[c] = -t[c]
    return t


E4 = e4_table()


def delta(conv):
    return 1 if conv == O.CONV_PAPER else 0


def quantise_row(x, conv):
    """(codes, bias as stored) of one row of float64 numbers."""
    amax = np.max(np.abs(x)) if not np.isnan(x).any() else np.nan
    most = 240.0 if conv == O.CONV_PAPER else 448.0
    if not np.isfinite(amax):
        bias, stored = 0, -128
    elif amax == 0:
        bias = stored = 0
    else:
        n = int(np.floor(np.log2(most / amax)))
        while amax * 2.0 ** n > most:
            n -= 1
        while amax * 2.0 ** (n + 1) <= most:
            n += 1
        bias = stored = max(-127, min(64, n))
    y = x * 2.0 ** (bias + delta(conv))
    a = np.clip(np.abs(y), 0, 448.0)
    grid = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    a = np.minimum(np.round(a / grid) * grid, 448.0)   # np.round: half to even
    codes = np.zeros(x.shape, np.uint8)
    ok = ~np.isnan(y)
    codes[ok] = np.searchsorted(E4[:127], a[ok]).astype(np.uint8)
    codes[~ok] = 0x7F
    codes |= (np.signbit(y) & ok).astype(np.uint8) << 7
    return codes, stored


def numbers(codes, bias, conv):
    """float64 numbers of codes [..., D] under stored biases [...]; rows marked non-finite are read under bias 0."""
    b = np.where(bias == -128, 0, bias.astype(np.int64))
    return E4[codes] * np.exp2(-(b + delta(conv)).astype(np.float64))[..., None]


def cached_rows(cache, table, b, positions):
    """Codes and biases [n, heads, D] / [n, heads] of a sequence's tokens, from numpy copies of the cache."""
    k8, v8, bk, bv = cache
    size = k8.shape[2]
    pages, off = table[b][positions // size], positions % size
    return k8[pages, :, off], bk[pages, :, off], v8[pages, :, off], bv[pages, :, off]


def attention(cache, table, q_start, kv_len, q, scale, causal, conv):
    """(out, lse, spread, score) in float64: spread = sum_j p_j |v_j| / sum_j p_j per output, score = the largest
    sum_i |q_i k_i| * |scale| over the keys a row sees (what its score errors are relative to)."""
    T, H, D = q.shape
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    spread, score = np.zeros((T, H, D)), np.zeros((T, H))
    hk = cache[0].shape[1]
    for b in range(len(kv_len)):
        first, n, length = q_start[b], q_start[b + 1] - q_start[b], kv_len[b]
        if n == 0 or length == 0:
            continue
        kc, kb, vc, vb = cached_rows(cache, table, b, np.arange(length))
        k, v = numbers(kc, kb, conv), numbers(vc, vb, conv)
        poison = (kb == -128) | (vb == -128)
        for h in range(H):
            g = h // (H // hk)
            for i in range(n):
                see = min(length, length - n + i + 1) if causal else length
                if see <= 0:
                    continue
                x = q[first + i, h]
                if poison[:see, g].any() or not np.isfinite(x).all():
                    out[first + i, h], lse[first + i, h] = np.nan, np.nan
                    continue
                s = k[:see, g] @ x * scale
                top = s.max()
                p = np.exp(s - top)
                lse[first + i, h] = top + np.log(p.sum())
                out[first + i, h] = p @ v[:see, g] / p.sum()
                spread[first + i, h] = p @ np.abs(v[:see, g]) / p.sum()
                score[first + i, h] = (np.abs(k[:see, g]) @ np.abs(x)).max() * abs(scale)
    return out, lse, spread, score


def make_case(seed, lens, news, heads, dim, page, conv, dtype=torch.bfloat16, spare=3, fill=None):
    """Random cache pages (codes without NaN unless `fill` is given for what no sequence owns), a shuffled page table and
    the batch's index tensors; everything on the CPU."""
    g = torch.Generator().manual_seed(seed)
    width = max(1, max(-(-n // page) for n in lens))
    owned = sum(-(-n // page) for n in lens)
    pages = owned + spare
    perm = torch.randperm(pages, generator=g)
    table = torch.zeros((len(lens), width), dtype=torch.int32)
    at = 0
    k8, v8 = (torch.randint(0, 256, (pages, heads, page, dim), generator=g, dtype=torch.uint8) for _ in range(2))
    k8[(k8 & 127) == 127] = 0x30
    v8[(v8 & 127) == 127] = 0x31
    # bytes uniform over the codes reach 448: biases around 7 to 10 make numbers of about one
    bk = torch.randint(6, 10, (pages, heads, page), generator=g, dtype=torch.int8)
    bv = torch.randint(5, 10, (pages, heads, page), generator=g, dtype=torch.int8)
    held = torch.zeros((pages, page), dtype=torch.bool)
    for b, n in enumerate(lens):
        need = -(-n // page)
        table[b, :need] = perm[at:at + need].to(torch.int32)
        for j in range(need):
            held[perm[at + j], :min(page, n - j * page)] = True
        at += need
    if fill is not None:
        stale = ~held
        k8.permute(0, 2, 1, 3)[stale] = fill
        v8.permute(0, 2, 1, 3)[stale] = fill
        bk.permute(0, 2, 1)[stale] = -128
        bv.permute(0, 2, 1)[stale] = -128
    q_start = torch.zeros(len(news) + 1, dtype=torch.int32)
    q_start[1:] = torch.tensor(news).cumsum(0)
    return dict(k8=k8, v8=v8, bk=bk, bv=bv, table=table, q_start=q_start, kv_len=torch.tensor(lens, dtype=torch.int32), g=g)
