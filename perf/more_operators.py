"""Operators at the head of a decoder and between its linears: what is measured, and the operators' plain forms.

  norm          y = norm(x + residual): layer norm or its root-mean-square form, with the sum, the statistics and, where an
                FP8 linear follows, E4 bytes of y under the scaling bias of its largest magnitude
  norm_bwd      the gradients of the sum, the weight and the additive vector
  logprobs      log probabilities of given tokens under softmax(scale * logits), the entropy of each row, its most probable
                tokens (equal logits: the lowest index first)
  logprobs_bwd  the gradient of the logits for gradients of log probabilities and entropies
  distill       per row, the divergence of a teacher's listed tokens from the student: "rest" false renormalises the listed
                ones, "rest" true treats everything that is not listed as one more outcome
  distill_bwd   its gradient for the student's logits

`run` with `own` false computes them from elementary torch operations in 32 bits; with `own` true it calls the library.
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _norm(op, name=None, **kw):
    c = {"op": op, "rows": 1, "cols": 4096, "dtype": "bf16", "kind": "layer", "residual": True, "shift": True, "bytes8": False,
         "paper": True}
    c.update(kw)
    if c["kind"] == "rms":
        c["shift"] = False
    if name is not None:
        c["name"] = name
    return c


def _loss(op, name=None, **kw):
    c = {"op": op, "rows": 1, "vocab": 32000, "pad": 0, "dtype": "bf16", "scale": 1.0, "banned": False}
    if op == "logprobs":
        c["top"] = 0
    if op.startswith("distill"):
        c.update(listed=32, rest=True)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One decoded token enters a layer of a 70B-shaped model: residual sum, norm, and the bytes that its QKV linear reads.
        _norm("norm", "norm_step1", rows=1, cols=8192, kind="rms", bytes8=True),
        # An 8192-token training batch of a 7B-shaped layer, the same fused into one call.
        _norm("norm", "norm_8192_bytes", rows=8192, cols=4096, bytes8=True),
        # Odd sizes in FP32 without a residual, as for an embedding of another width.
        _norm("norm", "norm_f32_odd", rows=1531, cols=1027, dtype="f32", residual=False),
        # The backward pass of that batch: the residual's gradient joins, the weight's gradient sums over 8192 rows.
        _norm("norm_bwd", "norm_bwd_8192", rows=8192, cols=4096),
        # A GPT-shaped micro batch in FP16, an odd number of tokens.
        _norm("norm_bwd", "norm_bwd_f16", rows=1021, cols=2048, dtype="f16"),
        # Serving: one token's log probability and the five most probable ones.
        _loss("logprobs", "logprobs_1", rows=1, vocab=32000, top=5),
        # Scoring a batch of 4096 evaluated tokens over a vocabulary of odd size.
        _loss("logprobs", "logprobs_4096", rows=4096, vocab=50257),
        # A teacher writes the twenty most probable tokens of 512 positions at temperature 2, from FP32 logits.
        _loss("logprobs", "logprobs_top20_f32", rows=512, vocab=128256, dtype="f32", scale=0.5, top=20, banned=True),
        # Fine-tuning by log probabilities with an entropy bonus.
        _loss("logprobs_bwd", "logprobs_bwd_4096", rows=4096, vocab=32000),
        # Distillation of a 2048-token batch from 64 listed tokens a position.
        _loss("distill", "distill_2048", rows=2048, vocab=32000, listed=64),
        # Its gradient, renormalised lists, FP16 logits of odd width.
        _loss("distill_bwd", "distill_bwd_f16", rows=2048, vocab=50257, listed=32, rest=False, scale=0.5, dtype="f16"),
        # A small classifier-sized head, FP32.
        _loss("distill_bwd", "distill_bwd_small", rows=37, vocab=1003, listed=8, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_bwd", "logprobs", "logprobs", "logprobs_bwd", "distill", "distill_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("norm"):
        cols = _log_int(rng, 64, 16384)
        if rng.random() < 0.7:
            cols = max(64, cols // 64 * 64)
        rows = _log_int(rng, 1, max(1, min(16384, 8192 * 4096 // (cols * (2 if dtype == "f32" else 1)))))
        kw = {"kind": rng.choice(["layer", "rms"]), "residual": rng.random() < 0.6}
        if op == "norm":
            kw["bytes8"] = rng.random() < 0.5
            kw["paper"] = rng.random() < 0.5
        return _norm(op, rows=rows, cols=cols, dtype=dtype, **kw)
    vocab = _log_int(rng, 1000, 131072)
    if rng.random() < 0.5:
        vocab = vocab // 16 * 16
    rows = _log_int(rng, 1, max(1, min(8192, 4096 * 32000 // (vocab * (2 if dtype == "f32" else 1)))))
    kw = {"rows": rows, "vocab": vocab, "dtype": dtype, "scale": rng.choice([1.0, 1.0, 0.5, 1.25]), "pad": rng.choice([0, 0, 0, 24]),
          "banned": rng.random() < 0.3}
    if op == "logprobs":
        kw["top"] = rng.choice([0, 1, _log_int(rng, 2, 32)])
    if op.startswith("distill"):
        kw["listed"], kw["rest"] = _log_int(rng, 4, 128), rng.random() < 0.5
    return _loss(op, **kw)


def work(case):
    size, rows = _SIZE[case["dtype"]], case["rows"]
    if case["op"] == "norm":
        n, cols = rows * case["cols"], case["cols"]
        per = size * (3 if case["residual"] else 1) + (1 if case["bytes8"] else size)
        stats = 8 if case["kind"] == "layer" else 4
        return {"bytes": n * per + rows * stats + cols * size * (2 if case["shift"] else 1), "flops": 10 * n}
    if case["op"] == "norm_bwd":
        n, cols = rows * case["cols"], case["cols"]
        stats = 8 if case["kind"] == "layer" else 4
        return {"bytes": n * size * (4 if case["residual"] else 3) + rows * stats + cols * size * (3 if case["shift"] else 2),
                "flops": 14 * n}
    n = rows * case["vocab"]
    if case["op"] == "logprobs":
        return {"bytes": n * size + rows * (8 + 8 + 12 * case["top"]), "flops": 7 * n}
    if case["op"] == "logprobs_bwd":
        return {"bytes": 2 * n * size + rows * (8 + 8 + 12), "flops": 7 * n}
    lists = rows * case["listed"] * 12
    if case["op"] == "distill":
        return {"bytes": n * size + lists + rows * 4, "flops": 5 * n}
    return {"bytes": 2 * n * size + lists + rows * 16, "flops": 5 * n}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
_EPS = 1e-5


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = dict(case)
    return (_prepare_norm if case["op"].startswith("norm") else _prepare_loss)(s, g, normal)


def _prepare_norm(s, g, normal):
    rows, cols, dt = s["rows"], s["cols"], _DTYPES[s["dtype"]]
    # the residual stream of a trained model: a few channels much larger than the others, a mean that is not zero
    gain = 1.0 + 20.0 * (torch.rand(cols, generator=g, device="cuda") < 0.005)
    stream = (normal(rows, cols) * gain + 0.1 * normal(cols)).to(dt)
    s["weight"] = (1.0 + 0.2 * normal(cols)).to(dt)
    s["vector"] = (0.1 * normal(cols)).to(dt) if s["shift"] else None
    if s["op"] == "norm":
        s["x"], s["res"] = ((0.5 * normal(rows, cols)).to(dt), stream) if s["residual"] else (stream, None)
        return s
    s["h"] = stream
    wide = stream.float()
    mean = wide.mean(-1, keepdim=True) if s["kind"] == "layer" else torch.zeros_like(wide[:, :1])
    s["rstd"] = (((wide - mean) ** 2).mean(-1) + _EPS) ** -0.5
    s["mean"] = mean.squeeze(-1).contiguous() if s["kind"] == "layer" else None
    s["dy"] = (1e-2 * normal(rows, cols)).to(dt)
    s["dh"] = (1e-2 * normal(rows, cols)).to(dt) if s["residual"] else None
    return s


def _prepare_loss(s, g, normal):
    rows, vocab, dt, scale = s["rows"], s["vocab"], _DTYPES[s["dtype"]], s["scale"]
    # rows from nearly decided to nearly undecided: a unit of noise, a row's own temperature, some tokens far ahead
    logits = torch.empty((rows, vocab + s["pad"]), dtype=dt, device="cuda")
    heat = 1.0 + 2.0 * torch.rand((rows, 1), generator=g, device="cuda")
    ahead = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
    step = max(1, (1 << 26) // vocab)
    for a in range(0, rows, step):
        x = normal(min(step, rows - a), vocab + s["pad"]) * heat[a:a + step]
        lead = heat[a:a + step] * (3.0 + 1.5 * normal(x.shape[0], 24))
        x.scatter_add_(1, ahead[a:a + step], lead)
        if s["banned"]:  # tokens that a grammar or a filter has ruled out
            x[torch.rand(x.shape, generator=g, device="cuda") < 0.05] = -math.inf
        logits[a:a + step] = x.to(dt)
    s["logits"] = logits[:, :vocab]
    if s["op"].startswith("logprobs"):
        # mostly one of the tokens ahead; a few positions are padding
        some = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        chance = torch.rand(rows, generator=g, device="cuda")
        t = torch.where(chance < 0.8, ahead[:, 0], some)
        if s["banned"]:  # a given token is one that may be given
            t = torch.where(torch.isinf(s["logits"].gather(1, t.unsqueeze(1)).squeeze(1)), s["logits"].float().argmax(-1), t)
        s["targets"] = torch.where(chance > 0.95, torch.full_like(t, -1), t) if rows > 8 else t
    else:
        # the teacher: the student's logits with noise, its most probable tokens, shorter lists for some positions
        k = s["listed"]
        s["index"] = torch.empty((rows, k), dtype=torch.int64, device="cuda")
        s["value"] = torch.empty((rows, k), dtype=torch.float32, device="cuda")
        for a in range(0, rows, step):
            z = s["logits"][a:a + step].float()
            z = scale * (z + 0.7 * normal(*z.shape))
            v, i = z.topk(k, -1)
            s["index"][a:a + step], s["value"][a:a + step] = i, v - torch.logsumexp(z, -1, keepdim=True)
        s["index"][(torch.rand((rows, 1), generator=g, device="cuda") < 0.1) & (torch.arange(k, device="cuda") >= k // 2)] = -1
    if s["op"].endswith("_bwd"):
        # what the forward pass leaves per row: the largest logit, ln sum exp(scale (x - largest)), the entropy, and the
        # second with the listed tokens left out
        s["saved"] = torch.zeros((rows, 4), dtype=torch.float32, device="cuda")
        for a in range(0, rows, step):
            top, logsum, p, lp = _softmax(s["logits"][a:a + step].float(), scale)
            keep = s["saved"][a:a + step]
            keep[:, 0], keep[:, 1] = top.squeeze(-1), logsum.squeeze(-1)
            keep[:, 2] = -(p * lp.clamp(min=-1e4)).sum(-1)
            if s["op"] == "distill_bwd":
                keep[:, 3] = _rest(p, s["index"][a:a + step]).log() + keep[:, 1]
        per_row = (32768.0 if s["dtype"] == "f16" else 1.0) / rows   # FP16 gradients come under a loss scale
        if s["op"] == "logprobs_bwd":
            s["g_logprob"] = -per_row * (0.5 + torch.rand(rows, generator=g, device="cuda"))
            s["g_entropy"] = torch.full((rows,), -0.01 * per_row, device="cuda")
        else:
            s["g_loss"] = per_row * (0.5 + torch.rand(rows, generator=g, device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2309_17224_b200 import fp8lin
    from paper_2309_17224_b200.module import default_context
    lib = default_context(0)
    if "out" not in s:  # the buffers that a training or serving loop keeps from step to step
        s["out"] = _buffers(s)
    o = s["out"]
    if s["op"] == "norm":
        lib.norm_fwd(s["x"], s["weight"], s["vector"], residual=s["res"], eps=_EPS, kind=_kind(fp8lin, s), h=o.get("h"), y=o.get("y"),
                     d_mean=o.get("mean"), d_rstd=o["rstd"], y8=o.get("y8"), d_amax_out=o.get("amax"), d_bias_out=o.get("bias"),
                     conv=fp8lin.CONV_PAPER if s["paper"] else fp8lin.CONV_NATIVE)
        return {k: v.view(torch.float8_e4m3fn) if k == "y8" else v for k, v in o.items()}
    if s["op"] == "norm_bwd":
        lib.norm_bwd(s["dy"], s["h"], s["weight"], s["mean"], s["rstd"], o["dx"], dh=s["dh"], dw=o["dw"], db=o.get("db"),
                     kind=_kind(fp8lin, s))
        return o
    if s["op"] == "logprobs":
        lib.token_logprobs(s["logits"], s["targets"], scale=s["scale"], logprob=o["logprob"], entropy=o["entropy"],
                           top_logprob=o.get("top_logprob"), top_index=o.get("top_index"))
        return o
    if s["op"] == "logprobs_bwd":
        lib.token_logprobs_bwd(s["logits"], s["targets"], s["saved"], o["dlogits"], g_logprob=s["g_logprob"],
                               g_entropy=s["g_entropy"], scale=s["scale"])
        return o
    if s["op"] == "distill":
        lib.distill_fwd(s["logits"], s["index"], s["value"], o["loss"], rest=s["rest"], scale=s["scale"])
        return o
    lib.distill_bwd(s["logits"], s["index"], s["value"], s["saved"], s["g_loss"], o["dlogits"], rest=s["rest"], scale=s["scale"])
    return o


def _kind(fp8lin, s):
    return fp8lin.NORM_LAYER if s["kind"] == "layer" else fp8lin.NORM_RMS


def _buffers(s):
    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    dt, rows = _DTYPES[s["dtype"]], s["rows"]
    if s["op"] == "norm":
        o = {"rstd": new(rows)}
        if s["kind"] == "layer":
            o["mean"] = new(rows)
        if s["residual"]:
            o["h"] = new(rows, s["cols"], dtype=dt)
        if s["bytes8"]:
            o.update(y8=new(rows, s["cols"], dtype=torch.uint8), amax=new(1), bias=new(1, dtype=torch.int32))
        else:
            o["y"] = new(rows, s["cols"], dtype=dt)
        return o
    if s["op"] == "norm_bwd":
        o = {"dx": new(rows, s["cols"], dtype=dt), "dw": new(s["cols"], dtype=dt)}
        if s["shift"]:
            o["db"] = new(s["cols"], dtype=dt)
        return o
    if s["op"] == "logprobs":
        o = {"logprob": new(rows), "entropy": new(rows)}
        if s["top"]:
            o.update(top_logprob=new(rows, s["top"]), top_index=new(rows, s["top"], dtype=torch.int64))
        return o
    if s["op"] == "distill":
        return {"loss": new(rows)}
    return {"dlogits": new(rows, s["vocab"], dtype=dt)}


def _pow2(n):
    """2^n for integers n in [-126, 127], exactly: the exponent field of a 32-bit number."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _run_plain(s):
    return {"norm": _norm_plain, "norm_bwd": _norm_bwd_plain, "logprobs": _logprobs_plain, "logprobs_bwd": _logprobs_bwd_plain,
            "distill": _distill_plain, "distill_bwd": _distill_bwd_plain}[s["op"]](s)


def _norm_plain(s):
    dt = _DTYPES[s["dtype"]]
    h = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(dt)
    d = h.float()
    o = {}
    if s["kind"] == "layer":
        mean = d.mean(-1, keepdim=True)
        d = d - mean
        o["mean"] = mean.squeeze(-1)
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + _EPS)
    y = d * rstd * s["weight"].float()
    if s["vector"] is not None:
        y = y + s["vector"].float()
    y = y.to(dt)
    o["rstd"] = rstd.squeeze(-1)
    if s["residual"]:
        o["h"] = h
    if not s["bytes8"]:
        o["y"] = y
        return o
    y = y.float()
    amax = y.abs().amax().view(1)
    mant, expo = torch.frexp(amax)                       # amax = mant * 2^expo, mant in [0.5, 1)
    top, lead = (7, 1.875) if s["paper"] else (8, 1.75)  # largest number of the format: lead * 2^top
    bias = top - (expo - 1) - (2 * mant > lead).to(expo.dtype)
    y8 = (y * _pow2(bias + (1 if s["paper"] else 0))).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    o.update(y8=y8, amax=amax, bias=bias)
    return o


def _norm_bwd_plain(s):
    dt = _DTYPES[s["dtype"]]
    xh, dy = s["h"].float(), s["dy"].float()
    if s["mean"] is not None:
        xh = xh - s["mean"].unsqueeze(-1)
    xh = xh * s["rstd"].unsqueeze(-1)
    o = {"dw": (dy * xh).sum(0).to(dt)}
    if s["vector"] is not None:
        o["db"] = dy.sum(0).to(dt)
    gy = dy * s["weight"].float()
    dx = gy - xh * (gy * xh).mean(-1, keepdim=True)
    if s["mean"] is not None:
        dx = dx - gy.mean(-1, keepdim=True)
    dx = dx * s["rstd"].unsqueeze(-1)
    o["dx"] = (dx if s["dh"] is None else dx + s["dh"].float()).to(dt)
    return o


def _softmax(x, scale):
    """Largest logit, ln sum exp(scale (x - largest)), probabilities and their logarithms."""
    top = x.amax(-1, keepdim=True)
    z = scale * (x - top)
    logsum = torch.exp(z).sum(-1, keepdim=True).log()
    lp = z - logsum
    return top, logsum, torch.exp(lp), lp


def _rest(p, index):
    """The probability of everything that a list does not hold (padding entries have index -1)."""
    valid = index >= 0
    hidden = torch.zeros_like(p, dtype=torch.bool)
    hidden.scatter_(1, torch.where(valid, index, index.amax(1, keepdim=True)), True)
    return p.masked_fill(hidden, 0.0).sum(-1)


def _logprobs_plain(s):
    x = s["logits"].float()
    _, _, p, lp = _softmax(x, s["scale"])
    given = s["targets"] >= 0
    o = {"logprob": torch.where(given, lp.gather(1, s["targets"].clamp(min=0).unsqueeze(1)).squeeze(1), torch.zeros_like(p[:, 0])),
         "entropy": -(p * lp.clamp(min=-1e4)).sum(-1)}
    if s["top"]:
        place = torch.arange(s["vocab"], device="cuda")
        index = []
        for _ in range(s["top"]):  # the lowest index among the largest that are left
            i = torch.where(x == x.amax(-1, keepdim=True), place, s["vocab"]).amin(-1, keepdim=True)
            x = x.scatter(1, i, -math.inf)
            index.append(i)
        o["top_index"] = torch.cat(index, 1)
        o["top_logprob"] = lp.gather(1, o["top_index"])
    return o


def _logprobs_bwd_plain(s):
    keep = s["saved"]
    lp = s["scale"] * (s["logits"].float() - keep[:, 0:1]) - keep[:, 1:2]
    p = torch.exp(lp)
    given = (s["targets"] >= 0).float()
    g, gh = (s["g_logprob"] * given).unsqueeze(1), s["g_entropy"].unsqueeze(1)
    d = -p * (g + gh * (lp.clamp(min=-1e4) + keep[:, 2:3]))
    d.scatter_add_(1, s["targets"].clamp(min=0).unsqueeze(1), g)
    return {"dlogits": (s["scale"] * d).to(s["logits"].dtype)}


def _teacher(s):
    """Which entries count, their probabilities, the probability of the rest, and the sum of both, in 64 bits."""
    valid = s["index"] >= 0
    v = s["value"].double().masked_fill(~valid, -math.inf)
    if not s["rest"]:
        return valid, torch.softmax(v, -1), None, torch.ones_like(v[:, 0])
    q = torch.exp(v)
    rest = (1.0 - q.sum(-1)).clamp(min=0.0)
    return valid, q, rest, q.sum(-1) + rest


def _distill_plain(s):
    _, _, p, lp = _softmax(s["logits"].float(), s["scale"])
    valid, q, rest, _ = _teacher(s)
    lp = lp.gather(1, s["index"].clamp(min=0)).double()
    loss = torch.where(valid, q * (q.log() - lp), torch.zeros_like(q)).sum(-1)
    if s["rest"]:
        loss = loss + torch.where(rest > 0, rest * (rest.log() - _rest(p, s["index"]).double().log()), torch.zeros_like(rest))
    return {"loss": loss.float()}


def _distill_bwd_plain(s):
    keep = s["saved"]
    p = torch.exp(s["scale"] * (s["logits"].float() - keep[:, 0:1]) - keep[:, 1:2])
    valid, q, rest, total = _teacher(s)
    index = torch.where(valid, s["index"], s["index"].amax(1, keepdim=True))
    others = total if rest is None else total - rest * torch.exp((keep[:, 1] - keep[:, 3]).double())
    d = p * others.float().unsqueeze(1)
    at = total.float().unsqueeze(1) * p.gather(1, index)
    d.scatter_(1, index, at)                             # a padding entry stands where a listed one does
    d.scatter_add_(1, index, -q.float().masked_fill(~valid, 0.0))
    return {"dlogits": (s["scale"] * s["g_loss"].unsqueeze(1) * d).to(s["logits"].dtype)}


# ---------------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits, a few rows at a time
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(s) if case["op"] == "norm" else _exact_norm_bwd(s)
    step = max(1, (1 << 25) // case["vocab"])
    parts = [_exact_rows(s, slice(a, min(a + step, case["rows"]))) for a in range(0, case["rows"], step)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _centred(h, layer):
    h = h.double()
    mean = h.sum(-1, keepdim=True) / h.shape[-1] if layer else torch.zeros_like(h[:, :1])
    dev = h - mean
    return mean.squeeze(-1), dev, (dev.pow(2).sum(-1, keepdim=True) / h.shape[-1] + _EPS).rsqrt()


def _exact_norm(s):
    dt = _DTYPES[s["dtype"]]
    h = s["x"] if s["res"] is None else (s["x"].double() + s["res"].double()).to(dt)   # statistics are of the stored sum
    mean, dev, rstd = _centred(h, s["kind"] == "layer")
    y = dev * rstd * s["weight"].double() + (0.0 if s["vector"] is None else s["vector"].double())
    o = {"rstd": rstd.squeeze(-1)}
    if s["kind"] == "layer":
        o["mean"] = mean
    if s["residual"]:
        o["h"] = h.double()
    if not s["bytes8"]:
        o["y"] = y
        return o
    y = y.to(dt).double()                                # bytes are those of y as it would be stored
    amax = float(y.abs().max())
    most = 240.0 if s["paper"] else 448.0
    n = math.floor(math.log2(most / amax))               # the largest integer n with amax * 2^n <= most
    while amax * 2.0 ** (n + 1) <= most:
        n += 1
    while amax * 2.0 ** n > most:
        n -= 1
    z = y * 2.0 ** (n + (1 if s["paper"] else 0))
    grid = 2.0 ** (torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    o["y8"] = (torch.round(z / grid) * grid).clamp(-448.0, 448.0)
    o["amax"] = torch.tensor([amax], dtype=torch.float64, device="cuda")
    o["bias"] = torch.tensor([n], dtype=torch.int32, device="cuda")
    return o


def _exact_norm_bwd(s):
    _, dev, rstd = _centred(s["h"], s["kind"] == "layer")
    xh, dy = dev * rstd, s["dy"].double()
    o = {"dw": (dy * xh).sum(0)}
    if s["vector"] is not None:
        o["db"] = dy.sum(0)
    gy = dy * s["weight"].double()
    n = xh.shape[-1]
    dx = rstd * (gy - xh * ((gy * xh).sum(-1, keepdim=True) / n))
    if s["kind"] == "layer":
        dx = dx - rstd * (gy.sum(-1, keepdim=True) / n)
    o["dx"] = dx if s["dh"] is None else dx + s["dh"].double()
    return o


def _exact_rows(s, at):
    z = s["scale"] * s["logits"][at].double()
    lse = torch.logsumexp(z, -1, keepdim=True)
    row = torch.arange(z.shape[0], device="cuda")
    if s["op"].startswith("logprobs"):
        t = s["targets"][at]
        given = t >= 0
        lp = z - lse
        entropy = -torch.where(lp > -math.inf, lp.exp() * lp, torch.zeros_like(lp)).sum(-1)
        if s["op"] == "logprobs":
            o = {"logprob": torch.where(given, lp[row, t.clamp(min=0)], torch.zeros_like(entropy)), "entropy": entropy}
            if s["top"]:
                o["top_index"] = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :s["top"]]
                o["top_logprob"] = lp.gather(1, o["top_index"])
            return o
        one = torch.zeros_like(lp)
        one[row[given], t[given]] = 1.0
        g = torch.where(given, s["g_logprob"][at].double(), torch.zeros_like(entropy)).unsqueeze(1)
        p = lp.exp()
        slope = torch.where(p > 0, p * (lp + entropy.unsqueeze(1)), torch.zeros_like(p))
        return {"dlogits": s["scale"] * (g * (one - p) - s["g_entropy"][at].double().unsqueeze(1) * slope)}
    p = (z - lse).exp()
    q = torch.zeros_like(p)
    listed_ = torch.zeros_like(p, dtype=torch.bool)
    loss = torch.zeros_like(p[:, 0])
    index, value = s["index"][at], s["value"][at].double()
    valid = index >= 0
    if not s["rest"]:
        norm = torch.logsumexp(value.masked_fill(~valid, -math.inf), -1, keepdim=True)
        value = value - norm
    r, c = valid.nonzero(as_tuple=True)
    q[r, index[r, c]] = value[r, c].exp()
    listed_[r, index[r, c]] = True
    terms = value[r, c].exp() * (value[r, c] - (z - lse)[r, index[r, c]])
    loss.index_add_(0, r, terms)
    grad = p * q.sum(-1, keepdim=True) - q
    if s["rest"]:
        q_rest = (1.0 - q.sum(-1)).clamp(min=0.0)
        p_rest = p.masked_fill(listed_, 0.0).sum(-1)
        loss = loss + torch.where(q_rest > 0, q_rest * (q_rest / p_rest).log(), torch.zeros_like(q_rest))
        grad = grad + q_rest.unsqueeze(1) * (p - p.masked_fill(listed_, 0.0) / p_rest.unsqueeze(1))
    if s["op"] == "distill":
        return {"loss": loss}
    return {"dlogits": s["scale"] * s["g_loss"][at].double().unsqueeze(1) * grad}
