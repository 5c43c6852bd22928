"""Serving operators on an FP8 key/value cache: what is measured, and the operators' plain forms.

Three operators share one cache of pages.  A page holds, per key/value head, `page` tokens of `head_dim` E4 bytes for
the keys and the same for the values, and one scaling bias (the integer of "floor(log2(max / amax))") per token and
head for each of the two:

  append  quantises the newest tokens' keys and values row by row (a row: one token, one head) into the pages
  read    gives tokens of the cache back as numbers
  attend  softmax(scale q k^T) v of each sequence's newest tokens over its cached tokens: one token a sequence
          (decode), a few (verification of drafted tokens), or a chunk of a prompt

`run` with `own` false computes them from elementary torch operations in 32 bits; with `own` true it calls the library.
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(op, name=None, **kw):
    c = {"op": op, "seqs": 1, "new": 1, "ctx": 1024, "ragged": True, "q_heads": 64, "kv_heads": 8, "head_dim": 128,
         "page": 64, "dtype": "bf16", "causal": True, "paper": True}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One decoding step of a 70B-shaped layer (64 query heads, 8 key/value heads) at the batch of 16: sixteen rows of
        # keys and values go into sixteen pages.  Pure latency.
        _case("append", "append_step16", seqs=16, new=1, ctx=2048, ragged=False, page=64),
        # Prompts of a GPT-shaped layer (32 heads of 64) whose QKV matmul left FP32: odd lengths, native bias convention.
        _case("append", "append_f32_odd", seqs=3, new=1531, ctx=1531, q_heads=32, kv_heads=32, head_dim=64, page=16,
              dtype="f32", paper=False),
        # A whole 8192-token batch of a 7B-shaped layer (32 heads of 128) enters the cache in one call.
        _case("append", "append_8192", seqs=4, new=2048, ctx=2048, ragged=False, q_heads=32, kv_heads=32, page=128),
        # One short sequence leaves the cache (to be moved, or checked) as bf16.
        _case("read", "read_777", seqs=1, new=777, ctx=777, page=32),
        # All tokens of sixteen sequences of up to 4096 come back.
        _case("read", "read_16x4096", seqs=16, new=4096, ctx=4096, page=64),
        # The smallest call of serving: one user, one new token, a context of about a thousand.
        _case("attend", "decode_1x1009", seqs=1, ctx=1009, page=16),
        # Sixteen users of a 70B-shaped model, contexts of 2048 to 4096 tokens.
        _case("attend", "decode_16x4096", seqs=16, ctx=4096, page=64),
        # A 7B-shaped model (every query head has keys of its own) with four long contexts: the cache is 270 MB.
        _case("attend", "decode_mha_4x8192", seqs=4, ctx=8192, q_heads=32, kv_heads=32, page=128),
        # Five drafted tokens a sequence are verified at once.
        _case("attend", "verify_16x5", seqs=16, new=5, ctx=2048, ragged=False, page=32),
        # Short prompts of a GPT-shaped model arrive in pieces of a few dozen tokens, odd sizes.
        _case("attend", "chunk_gpt_odd", seqs=5, new=37, ctx=701, q_heads=32, kv_heads=32, head_dim=64, page=16,
              paper=False),
        # Four users' prompts in chunks of up to 256 tokens over contexts of up to 4096.
        _case("attend", "chunk_4x256", seqs=4, new=256, ctx=4096, page=64),
        # The last 2048 tokens (the prefill batch) of a 16384-token prompt.
        _case("attend", "chunk_2048_16k", seqs=1, new=2048, ctx=16384, page=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    q_heads, kv_heads, head_dim = rng.choice([(64, 8, 128), (64, 8, 128), (32, 32, 128), (32, 32, 64), (16, 16, 128), (16, 2, 64),
                                              (40, 8, 128)])
    kw = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]),
              paper=rng.random() < 0.5, ragged=rng.random() < 0.75)
    if op == "attend":
        kind = rng.choice(["decode", "decode", "few", "chunk", "chunk"])
        kw["new"] = 1 if kind == "decode" else _log_int(rng, 2, 16) if kind == "few" else _log_int(rng, 17, 2048)
        kw["seqs"] = _log_int(rng, 1, 64) if kind != "chunk" else _log_int(rng, 1, 8)
        kw["causal"] = rng.random() < 0.85
        most = 16384
        while True:  # within the largest listed cases, in cached bytes and in products
            kw["ctx"] = max(_log_int(rng, 64, most), kw["new"])
            c = _case(op, **kw)
            if (c["seqs"] * c["ctx"] * kv_heads * head_dim <= 4 * 8192 * 32 * 128
                    and c["seqs"] * c["new"] * c["ctx"] * q_heads * head_dim <= 2048 * 15360 * 64 * 128):
                return c
            kw["seqs"], kw["new"], most = max(1, kw["seqs"] // 2), max(1, kw["new"] * 2 // 3) if kind != "decode" else 1, most * 3 // 4
    kw["dtype"] = rng.choice(["bf16", "bf16", "f32", "f16"])
    rows = _log_int(rng, 1, 32768 // kv_heads * 8)
    kw["seqs"] = min(rows, _log_int(rng, 1, 32))
    kw["new"] = max(1, rows // kw["seqs"])
    kw["ctx"] = kw["new"] + rng.choice([0, 0, 1, 77])
    return _case(op, **kw)


def _lengths(case):
    """(new tokens, cached tokens with the new ones) of every sequence; the first sequence has the largest of both."""
    r = random.Random("%(seqs)d %(new)d %(ctx)d" % case)
    full = not case["ragged"]
    new = [case["new"] if full or i == 0 else r.randint(max(1, case["new"] // 2), case["new"]) for i in range(case["seqs"])]
    ctx = [case["ctx"] if full or i == 0 else r.randint(max(n, case["ctx"] // 2), case["ctx"]) for i, n in enumerate(new)]
    return new, ctx


def work(case):
    new, ctx = _lengths(case)
    tokens, d, hk, hq = sum(new), case["head_dim"], case["kv_heads"], case["q_heads"]
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] != "attend":  # numbers on one side, bytes and biases on the other
        return {"bytes": 2 * tokens * hk * (d * (size + 1) + 1), "flops": 0}
    # with a causal mask the new token i of a sequence sees ctx - new + 1 + i tokens
    seen = sum(n * c - n * (n - 1) // 2 if case["causal"] else n * c for n, c in zip(new, ctx))
    return {"bytes": 2 * sum(ctx) * hk * (d + 1) + tokens * hq * (2 * size * d + 4), "flops": 4 * seen * hq * d}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _pow2(n):
    """2^n for integers n in [-126, 127], exactly: the exponent field of a 32-bit number."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise_rows(x, paper):
    """E4 bytes (as float8 values) and biases of the rows of `x` (last dimension): the plain form of append."""
    x = x.float()
    amax = x.abs().amax(-1)
    mant, expo = torch.frexp(amax)                       # amax = mant * 2^expo, mant in [0.5, 1)
    top, lead = (7, 1.875) if paper else (8, 1.75)       # largest number of the format: lead * 2^top
    bias = top - (expo - 1) - (2 * mant > lead).to(expo.dtype)
    bias = torch.where(amax > 0, bias, torch.zeros_like(bias)).clamp(-127, 64)
    y = (x * _pow2(bias + (1 if paper else 0)).unsqueeze(-1)).clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn), bias.to(torch.int8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, ctx = _lengths(case)
    seqs, hq, hk, d, page = (case[k] for k in ("seqs", "q_heads", "kv_heads", "head_dim", "page"))
    tokens, per_seq = sum(new), -(-case["ctx"] // page)
    pages = seqs * per_seq + 7                           # a few pages of the pool belong to nobody
    dev = {"device": "cuda"}
    s = {"op": case["op"], "paper": case["paper"], "causal": case["causal"], "max_new": case["new"], "max_ctx": case["ctx"]}
    s["table"] = torch.randperm(pages, generator=g, **dev)[:seqs * per_seq].to(torch.int32).view(seqs, per_seq)
    s["start"] = torch.tensor([sum(new[:i]) for i in range(seqs + 1)], dtype=torch.int32, **dev)
    s["ctx"] = torch.tensor(ctx, dtype=torch.int32, **dev)
    # keys and values: unit normal, a few channels of the keys several times larger, as projections of a trained model have
    s["k8"], s["v8"] = (torch.empty((pages, hk, page, d), dtype=torch.uint8, **dev) for _ in range(2))
    s["bk"], s["bv"] = (torch.empty((pages, hk, page), dtype=torch.int8, **dev) for _ in range(2))
    gain = 1.0 + 5.0 * (torch.rand((hk, 1, d), generator=g, **dev) < 0.02)
    step = max(1, (1 << 26) // (hk * page * d))
    for a in range(0, pages, step):
        for t8, tb, scale in ((s["k8"], s["bk"], gain), (s["v8"], s["bv"], 1.0)):
            x = torch.randn((min(step, pages - a), hk, page, d), generator=g, **dev) * scale
            codes, bias = _quantise_rows(x.to(torch.bfloat16), case["paper"])
            t8[a:a + step], tb[a:a + step] = codes.view(torch.uint8), bias
    # what the QKV matmul leaves: queries, keys and values of a token side by side in one row
    if case["op"] != "read":
        qkv = torch.randn((tokens, hq + 2 * hk, d), generator=g, **dev)
        qkv[:, hq:hq + hk] *= gain.view(1, hk, d)
        qkv = qkv.to(_DTYPES[case["dtype"]])
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        s["shape"], s["dtype"] = (tokens, hk, d), _DTYPES[case["dtype"]]
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2309_17224_b200 import fp8lin
    from paper_2309_17224_b200.module import default_context
    if "cache" not in s:  # the handles that a serving program makes with its cache and its batch
        s["cache"] = fp8lin.KvCache(s["k8"], s["v8"], s["bk"], s["bv"],
                                    conv=fp8lin.CONV_PAPER if s["paper"] else fp8lin.CONV_NATIVE)
        s["batch"] = fp8lin.SeqBatch(s["start"], s["ctx"], s["table"], max_q_len=s["max_new"], max_kv_len=s["max_ctx"])
    lib = default_context(0)
    if s["op"] == "append":
        lib.kv_append(s["cache"], s["batch"], s["k"], s["v"])
        return s["k8"].view(torch.float8_e4m3fn), s["v8"].view(torch.float8_e4m3fn), s["bk"], s["bv"]
    if s["op"] == "read":
        k, v = (torch.empty(s["shape"], dtype=s["dtype"], device="cuda") for _ in range(2))
        lib.kv_read(s["cache"], s["batch"], k, v)
        return k, v
    q = s["q"]
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    lib.attn_paged(s["cache"], s["batch"], q, out, causal=s["causal"], lse=lse)
    return out, lse


def _places(s, tokens):
    """Of every new token: its sequence, its index among the sequence's new ones, its page and its place in the page."""
    t = torch.arange(tokens, device="cuda")
    seq = (t.unsqueeze(1) >= s["start"][1:].unsqueeze(0)).sum(1)
    first, count = s["start"][seq], s["start"][seq + 1] - s["start"][seq]
    index = t - first
    pos = s["ctx"][seq] - count + index
    page = s["k8"].shape[2]
    return seq, index, s["table"][seq, pos // page].long(), pos % page


def _numbers(codes, bias, paper):
    """The numbers that E4 bytes stand for, in 32 bits."""
    return codes.view(torch.float8_e4m3fn).float() * _pow2(-(bias.int() + (1 if paper else 0))).unsqueeze(-1)


def _run_plain(s):
    if s["op"] == "append":
        _, _, page, off = _places(s, s["k"].shape[0])
        (kc, kb), (vc, vb) = _quantise_rows(s["k"], s["paper"]), _quantise_rows(s["v"], s["paper"])
        s["k8"][page, :, off], s["v8"][page, :, off] = kc.view(torch.uint8), vc.view(torch.uint8)
        s["bk"][page, :, off], s["bv"][page, :, off] = kb, vb
        return s["k8"].view(torch.float8_e4m3fn), s["v8"].view(torch.float8_e4m3fn), s["bk"], s["bv"]
    if s["op"] == "read":
        _, _, page, off = _places(s, s["shape"][0])
        return (_numbers(s["k8"][page, :, off], s["bk"][page, :, off], s["paper"]).to(s["dtype"]),
                _numbers(s["v8"][page, :, off], s["bv"][page, :, off], s["paper"]).to(s["dtype"]))
    q, table = s["q"], s["table"].long()
    tokens, hq, d = q.shape
    seqs, per_seq = table.shape
    hk, page = s["k8"].shape[1:3]
    group, most, width = hq // hk, s["max_new"], per_seq * page
    k, v = (_numbers(s[c][table], s[b][table], s["paper"]).transpose(1, 2).reshape(seqs, hk, width, d)
            for c, b in (("k8", "bk"), ("v8", "bv")))
    first, count = s["start"][:-1], s["start"][1:] - s["start"][:-1]
    i = torch.arange(most, device="cuda")
    rows = (first.unsqueeze(1) + i).clamp(max=tokens - 1)                      # short sequences repeat a row, dropped below
    qp = q[rows].float().view(seqs, most, hk, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hk, group * most, d)
    score = torch.matmul(qp, k.transpose(2, 3)).view(seqs, hk, group, most, width) * (1.0 / math.sqrt(d))
    j = torch.arange(width, device="cuda")
    seen = (j < s["ctx"].view(-1, 1, 1)).expand(seqs, most, width)
    if s["causal"]:
        seen = seen & (j <= (s["ctx"] - count).view(-1, 1, 1) + i.view(1, -1, 1))
    score = score.masked_fill(~seen.view(seqs, 1, 1, most, width), -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(seqs, hk, group * most, width), v).view(seqs, hk, group, most, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = (top + torch.log(total)).squeeze(-1)
    seq, index, _, _ = _places(s, tokens)
    return (out.permute(0, 3, 1, 2, 4)[seq, index].reshape(tokens, hq, d).to(q.dtype),
            lse.permute(0, 3, 1, 2)[seq, index].reshape(tokens, hq))


# ---------------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------------
def _two_to(n):
    """2^n in 64 bits, exactly (a power function is off in the last place, which would break ties)."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4_table():
    """The numbers of the 256 E4M3 bytes (sign, four exponent bits of bias 7, three mantissa bits)."""
    b = torch.arange(256, device="cuda", dtype=torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * _two_to(e - 10))
    return torch.where(b >= 128, -mag, mag)


def exact(case, seed):
    s = prepare(case, seed)
    new, ctx = _lengths(case)
    page, shift = case["page"], 1 if case["paper"] else 0
    decode = _e4_table()
    at = 0
    if case["op"] == "append":
        k8, v8 = decode[s["k8"].long()], decode[s["v8"].long()]
        most = 240.0 if case["paper"] else 448.0
        for b in range(case["seqs"]):
            pos = torch.arange(ctx[b] - new[b], ctx[b], device="cuda")
            pages, off = s["table"][b].long()[pos // page], pos % page
            for x, codes, biases in ((s["k"], k8, s["bk"]), (s["v"], v8, s["bv"])):
                x = x[at:at + new[b]].double()
                amax = x.abs().amax(-1)
                # the largest integer n with amax * 2^n <= most: an estimate from the logarithm, corrected by products
                n = torch.floor(torch.log2(most / amax.clamp(min=1e-60)))
                n = n - (amax * _two_to(n) > most).double()
                n = n + (amax * _two_to(n + 1) <= most).double()
                n = torch.where(amax > 0, n, torch.zeros_like(n)).clamp(-127, 64)
                y = x * _two_to(n + shift).unsqueeze(-1)
                grid = _two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                codes[pages, :, off] = (torch.round(y / grid) * grid).clamp(-448.0, 448.0)
                biases[pages, :, off] = n.to(torch.int8)
            at += new[b]
        return k8, v8, s["bk"], s["bv"]
    hk, d = case["kv_heads"], case["head_dim"]

    def tokens_of(b, a, z):
        pos = torch.arange(a, z, device="cuda")
        pages, off = s["table"][b].long()[pos // page], pos % page
        return [decode[s[c][pages, :, off].long()] / _two_to(s[n][pages, :, off].long() + shift).unsqueeze(-1)
                for c, n in (("k8", "bk"), ("v8", "bv"))]

    if case["op"] == "read":
        both = [tokens_of(b, ctx[b] - new[b], ctx[b]) for b in range(case["seqs"])]
        return torch.cat([x[0] for x in both]), torch.cat([x[1] for x in both])
    group = case["q_heads"] // hk
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        k, v = tokens_of(b, 0, ctx[b])
        hidden = None
        if case["causal"]:
            last = torch.arange(ctx[b] - new[b], ctx[b], device="cuda")
            hidden = torch.arange(ctx[b], device="cuda").unsqueeze(0) > last.unsqueeze(1)
        for h in range(case["q_heads"]):
            score = s["q"][at:at + new[b], h].double() @ k[:, h // group].t() / math.sqrt(d)
            if hidden is not None:
                score.masked_fill_(hidden, -math.inf)
            lse[at:at + new[b], h] = torch.logsumexp(score, -1)
            out[at:at + new[b], h] = torch.softmax(score, -1) @ v[:, h // group]
        at += new[b]
    return out, lse
