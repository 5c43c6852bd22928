"""Token log probabilities and distillation against the definitions in 64 bits.

Tolerances count FP32 roundings U = 2^-24.  With d = (x - m) * scale * log2 e: a term 2^d is off by 3 U |d| ln 2 from d and by
2^-22 from the exponential; a sum's terms are joined in at most n / 2T + 24 additions and as many changes of the maximum as
a thread meets vectors (n / 8T at most, each one more exponential), T the threads of a row: 128 at least, 64 of many rows.  So ln sum is off by SUM(n) + 2^-22 * E, E the mean of
(largest z - z), and a log probability by that and 4 U times its size."""
import math

import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin


@pytest.fixture(scope="module")
def ctx(L):
    return L.Context(0)


def new(*shape, dtype=F32):
    t = torch.empty(shape, dtype=dtype, device="cuda")
    return t.view(torch.uint8).fill_(0xA5).view(dtype).view(shape) if t.numel() else t


def logits_of(rows, vocab, dtype, seed, spread=2.0, ld=None, first=0):
    """Rows `ld` apart that begin `first` elements behind a 16-byte boundary."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = ld or vocab
    flat = torch.empty(rows * ld + first + 64, dtype=dtype, device="cuda")
    x = flat[first:].as_strided((rows, vocab), (ld, 1))
    x.copy_(torch.randn((rows, vocab), generator=g, device="cuda") * spread)
    return x


def log_error(lp, z_scale, threads=128):
    """Bound of |error of ln sum|, per row: 64-bit log probabilities in, see above."""
    n = lp.shape[-1]
    p = lp.exp()
    lead = lp.amax(-1, keepdim=True)
    far = torch.where(p > 0, p * (lead - lp), torch.zeros_like(p)).sum(-1)
    return (n / (2 * threads) + 24) * U + (n / (8 * threads) + 16) * 2.0 ** -22 + 2.0 ** -22 * far


def near(got, want, bound):
    """Equal where not finite, within the bound elsewhere."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest])
    bound = bound.expand_as(want) if torch.is_tensor(bound) else torch.full_like(want, bound)
    off = (got - want).abs()
    assert bool((off[fine] <= bound[fine]).all()), (float(off[fine].max()), float((off[fine] / bound[fine]).max()))


def check_tokens(ctx, x, targets, scale, k, itype=torch.int64, threads=128):
    rows, vocab = x.shape
    out = {n: new(rows) for n in ("logprob", "entropy", "lse")}
    saved, top_lp, top_i = new(rows, 4), new(rows, k) if k else None, new(rows, k, dtype=itype) if k else None
    ctx.token_logprobs(x, targets, scale=scale, saved=saved, top_logprob=top_lp, top_index=top_i, **out)
    lp, lse = R.log_softmax(x, scale)
    err = log_error(lp, scale, threads)
    given = (targets >= 0) & (targets < vocab)
    want = torch.where(given, lp.gather(1, targets.clamp(0, vocab - 1).long().unsqueeze(1)).squeeze(1), torch.zeros_like(lse))
    want = torch.where(targets >= vocab, torch.full_like(want, NAN), want)
    near(out["logprob"], want, err + 4 * U * want.abs().nan_to_num(0, 0, 0))
    near(out["lse"], lse, err + 3 * U * (scale * x.double().abs().nan_to_num(0, 0, 0)).amax(-1) + U * lse.abs().nan_to_num(0, 0, 0))
    h = R.entropy(lp)
    near(out["entropy"], h, (err + 8 * U) * (2 + 2 * h))
    if k:
        index = R.top(x, k)
        assert torch.equal(top_i.long(), index)
        want = lp.gather(1, index)
        near(top_lp, want, (err.unsqueeze(1) + 4 * U * want.abs().nan_to_num(0, 0, 0)))
    return saved, lp


VOCABS = [1, 2, 7, 8, 9, 31, 64, 257, 1000, 1003, 2047, 4096, 5003, 32000, 50257, 70001]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_tokens(ctx, vocab, dtype):
    for rows, ld, first, scale, k, itype in ((5, vocab, 0, 1.0, min(vocab, 5), torch.int64), (3, vocab + 5, 1, 0.5, min(vocab, 128), torch.int32),
                                             (1, vocab, 3, 1.5, min(vocab, 20), torch.int64), (2, vocab + 8, 0, 1.0, 0, torch.int32)):
        x = logits_of(rows, vocab, dtype, vocab + rows, ld=ld, first=first)
        targets = torch.arange(rows, device="cuda", dtype=itype) * 7919 % vocab
        if rows > 2:
            targets[1] = -1
        check_tokens(ctx, x, targets, scale, k, itype)
    assert ctx.device_flags() == 0


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [9, 1003, 32000])
def test_masked_rows(ctx, vocab, dtype):
    """Masks of -infinity and of the type's lowest value: some tokens, all but one, all but two, all."""
    low = torch.finfo(dtype).min
    x = logits_of(8, vocab, dtype, vocab)
    keep = torch.tensor([2, vocab - 1], device="cuda")
    x[0, ::3] = -INF
    for r, value, left in ((1, -INF, 1), (2, -INF, 2), (3, -INF, 0), (4, low, 1), (5, low, 2), (6, low, 0)):
        own = x[r, keep[:left]].clone()
        x[r] = value
        x[r, keep[:left]] = own
    x[7, 1:] = -INF                                          # the first token is the only one, and it is the lowest number
    x[7, 0] = low
    for target in (2, 0, vocab - 1):
        check_tokens(ctx, x, torch.full((8,), target, device="cuda"), 1.0, min(vocab, 40))
    assert ctx.device_flags() == 0


def test_rows_that_are_no_numbers(ctx, L):
    for dtype in (BF16, F16, F32):
        for vocab in (40, 1003, 8192):
            x = logits_of(6, vocab, dtype, 3)
            x[1, 5], x[2, vocab - 1], x[3, 0], x[4, 7] = NAN, INF, NAN, INF
            x[4, 8] = -INF
            out = [new(6) for _ in range(3)]
            top_lp, top_i, saved = new(6, 3), new(6, 3, dtype=torch.int32), new(6, 4)
            t = torch.full((6,), 9, dtype=torch.int32, device="cuda")
            ctx.token_logprobs(x, t, logprob=out[0], entropy=out[1], lse=out[2], saved=saved, top_logprob=top_lp, top_index=top_i)
            bad = torch.tensor([False, True, True, True, True, False], device="cuda")
            for o in (*out, *top_lp.unbind(1)):
                assert torch.equal(torch.isnan(o), bad)
            assert bool((top_i[bad] == -1).all()) and torch.equal(top_i[~bad].long(), R.top(x[~bad], 3))
            dx = new(6, vocab, dtype=dtype)
            ctx.token_logprobs_bwd(x, t, saved, dx, g_logprob=torch.ones(6, device="cuda"))
            assert torch.equal(torch.isnan(dx).all(1), bad) and not bool(torch.isnan(dx[~bad]).any())


def test_equal_and_ordered_logits(ctx):
    """Ties go to the lowest index, -0 ties with 0; rows that pass the buffer of candidates, in rising, falling and equal order."""
    for vocab in (64, 3000, 32000, 50257):
        x = torch.zeros((7, vocab), device="cuda")
        x[1, 1::2] = -0.0
        x[2] = torch.arange(vocab, device="cuda") / 64
        x[3] = -x[2]
        x[4] = torch.arange(vocab, device="cuda") % 5
        x[5, vocab // 2:] = 1.0
        x[6, -40:] = torch.arange(40, device="cuda") % 2
        for dtype in (F32, BF16):
            for k in (1, 33, 64, min(vocab, 128)):
                top_lp, top_i = new(7, k), new(7, k, dtype=torch.int64)
                ctx.token_logprobs(x.to(dtype), top_logprob=top_lp, top_index=top_i)
                assert torch.equal(top_i, R.top(x.to(dtype), k))


def test_given_tokens_outside_the_vocabulary(ctx, L):
    x = logits_of(4, 100, BF16, 4)
    ctx.device_flags()
    for itype in (torch.int32, torch.int64):
        t = torch.tensor([99, 100, -1, torch.iinfo(itype).max], dtype=itype, device="cuda")
        saved, _ = check_tokens(ctx, x, t, 1.0, 0, itype)
        assert ctx.device_flags() == L.FLAG_BAD_INDEX
        dx = new(4, 100, dtype=BF16)
        ctx.token_logprobs_bwd(x, t, saved, dx, g_logprob=torch.ones(4, device="cuda"))
        assert ctx.device_flags() == L.FLAG_BAD_INDEX and bool((dx[1:] == 0).all()) and bool((dx[0] != 0).any())


def check_gradient(got, want, size, err, dtype):
    """`size`: magnitudes of what the gradient is a sum of; `err`: relative error of a probability."""
    near(got, want.to(dtype).double() if not bool(torch.isfinite(want).all()) else want,
         size * (err.unsqueeze(1) + 2.0 ** -20) + want.abs() * R.HALF[dtype] + R.TINY[dtype])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [1, 7, 64, 1003, 8192, 32000, 50257])
def test_token_gradient(ctx, vocab, dtype):
    for rows, ld, first, scale, masked in ((6, vocab, 0, 1.0, False), (6, vocab + 5, 1, 0.7, True), (2, vocab, 5, 1.5, True)):
        x = logits_of(rows, vocab, dtype, vocab + rows, ld=ld, first=first)
        if masked and vocab > 2:
            x[0, ::3] = -INF
            x[1] = -INF
        t = torch.arange(rows, device="cuda") * 7919 % vocab
        if rows > 2:
            t[2] = -1
            x[3, t[3]] = 30.0                                     # nearly certain
        saved, lp = check_tokens(ctx, x, t, scale, 0)
        g = torch.Generator(device="cuda").manual_seed(vocab)
        gl, gh = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
        if rows > 4:
            gl[4] = gh[4] = 0.0
        p, h = lp.exp(), R.entropy(lp).unsqueeze(1)
        lean = torch.where(p > 0, p * (1 + lp.abs() + h), torch.zeros_like(p))
        for a, b in ((gl, gh), (gl, None), (None, gh), (gl[:1].expand(rows), gh[:1].expand(rows))):
            dx, amax = new(rows, vocab, dtype=dtype), new(1)
            ctx.token_logprobs_bwd(x, t, saved, dx, g_logprob=a, g_entropy=b, scale=scale, d_amax=amax)
            want = R.token_grad(x, t, a, b, scale)
            size = scale * lean * ((0 if a is None else a.double().abs()) + (0 if b is None else b.double().abs())).unsqueeze(1)
            size = size.scatter_add(1, t.clamp(min=0).unsqueeze(1), torch.full_like(size[:, :1], 2.0 ** -3) * (0 if a is None else a.double().abs().unsqueeze(1)) * scale * (1 - p.gather(1, t.clamp(min=0).unsqueeze(1))))
            check_gradient(dx, want, size, 4 * log_error(lp, scale) + 8 * U * 64, dtype)
            assert float(amax) == float(dx.float().abs().max())
        # other alignment, other distance, the logits' own place
        wide = new(rows, vocab + 3, dtype=dtype)[:, 1:vocab + 1]
        ctx.token_logprobs_bwd(x, t, saved, dx, g_logprob=gl, g_entropy=gh, scale=scale)
        ctx.token_logprobs_bwd(x, t, saved, wide, g_logprob=gl, g_entropy=gh, scale=scale)
        assert torch.equal(dx, wide)
        ctx.token_logprobs_bwd(x, t, saved, x, g_logprob=gl, g_entropy=gh, scale=scale)
        assert torch.equal(x, dx)


def teacher(rows, vocab, listed, seed, x, scale, itype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = scale * (x.float().nan_to_num(0, 0, -50.0) + torch.randn((rows, vocab), generator=g, device="cuda"))
    value, index = torch.log_softmax(z, -1).topk(listed, -1)
    return index.to(itype), value.contiguous()


def check_distill(ctx, x, index, value, rest, scale, dtype, threads=128, pick=slice(None)):
    rows, vocab = x.shape
    loss, saved, dx, amax = new(rows), new(rows, 4), new(rows, vocab, dtype=dtype), new(1)
    ctx.distill_fwd(x, index, value, loss, rest=rest, scale=scale, saved=saved)
    some = x[pick], index[pick], value[pick]   # the rows that are compared
    want, grad = R.distill(*some, rest, scale)
    lp, _ = R.log_softmax(some[0], scale)
    p = lp.exp()
    err = 4 * log_error(lp, scale, threads) + 64 * U
    # terms q (ln q - lp): sizes of the parts, each off by err and 4 U of its size; q_r ln q_r by 2^-24 of q_r's logarithm
    reach = torch.where(torch.isfinite(some[2]), some[2].abs(), torch.zeros_like(some[2])).double().amax(-1) + 1
    far = lp.clamp(min=-700).gather(1, some[1].long().clamp(0, vocab - 1)).abs().amax(-1)
    near(loss[pick], want, (err + 8 * U * (reach + far + 30)) * 2)
    plain = new(rows)
    ctx.distill_fwd(x, index, value, plain, rest=rest, scale=scale)
    assert torch.equal(plain, loss) or bool(torch.isnan(loss).any())
    g = torch.Generator(device="cuda").manual_seed(vocab)
    gl = torch.rand(rows, generator=g, device="cuda") + 0.5
    for up in (gl, gl[:1].expand(rows)):
        ctx.distill_bwd(x, index, value, saved, up, dx, rest=rest, scale=scale, d_amax=amax)
        full = up[pick].double().unsqueeze(1) * grad
        q = torch.zeros_like(p)
        for r in range(len(want)):
            for j, (a, _) in R.teacher_of(some[1][r].tolist(), some[2][r].tolist(), vocab, rest)[0].items():
                q[r, j] = a
        left = (1 - q.sum(-1, keepdim=True)).clamp(min=0) if rest else torch.zeros_like(p[:, :1])
        others = torch.where(q > 0, torch.zeros_like(p), p)
        spread = left * others / others.sum(-1, keepdim=True).clamp(min=1e-300)
        size = up[pick].double().unsqueeze(1) * scale * (p + q + spread)
        finite = torch.isfinite(full).all(1)
        check_gradient(dx[pick][finite], full[finite], size[finite], err[finite], dtype)
        assert float(amax) == float(dx.float().abs().max()) or bool(torch.isnan(dx).any())
    return saved, dx


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab,listed", [(1, 1), (9, 3), (64, 64), (1003, 8), (4096, 64), (32000, 64), (50257, 33), (70001, 256)])
def test_distillation(ctx, vocab, listed, dtype, rest):
    for rows, ld, first, scale, itype in ((5, vocab, 0, 1.0, torch.int64), (3, vocab + 5, 1, 0.5, torch.int32), (1, vocab + 8, 4, 1.25, torch.int64)):
        x = logits_of(rows, vocab, dtype, vocab + rows, ld=ld, first=first)
        index, value = teacher(rows, vocab, listed, vocab, x, scale, itype)
        saved, dx = check_distill(ctx, x, index, value, rest, scale, dtype)
        # lists with a gap between their rows, other alignment of the gradient, the logits' own place
        wide_i, wide_v = new(rows, listed + 3, dtype=itype), new(rows, listed + 5)
        wide_i[:, :listed], wide_v[:, :listed] = index, value
        g = torch.rand(rows, device="cuda")
        ctx.distill_bwd(x, index, value, saved, g, dx, rest=rest, scale=scale)
        other = new(rows, vocab + 3, dtype=dtype)[:, 1:vocab + 1]
        ctx.distill_bwd(x, wide_i[:, :listed], wide_v[:, :listed], saved, g, other, rest=rest, scale=scale)
        assert torch.equal(dx, other)
        ctx.distill_bwd(x, index, value, saved, g, x, rest=rest, scale=scale)
        assert torch.equal(x, dx)
    assert ctx.device_flags() == 0


@pytest.mark.parametrize("rest", [True, False])
def test_odd_lists(ctx, L, rest):
    """Padding, the same token twice, no token, q = 0, no entry that counts, everything listed, sums above 1, tokens that the
    student rules out, a student far from the rest."""
    for vocab in (40, 1003):
        x = logits_of(12, vocab, F32, 7)
        index, value = teacher(12, vocab, 8, 8, x, 1.0)
        index[0, 2], index[1, 3:] = -1, -1
        index[2, 5], index[3, 1:4] = index[2, 1], index[3, 0]
        index[4] = -1
        value[5, 3] = -INF
        value[6] = -INF
        value[7] = -1.0                                             # a sum of 2.9
        x[8, index[8, 4]] = -INF                                    # the student rules a listed token out
        keep = x[9, index[9]].clone()
        x[9] = -INF                                                 # ... and here every other one
        x[9, index[9]] = keep
        x[10, index[10]] += 150.0                                   # the rest is 1e-65: no FP32 number, its logarithm is one
        x[11] = -INF
        ctx.device_flags()
        check_distill(ctx, x, index, value, rest, 1.0, F32)
        assert ctx.device_flags() == 0
        index[0, 2] = vocab
        check_distill(ctx, x, index, value, rest, 1.0, F32)
        assert ctx.device_flags() == L.FLAG_BAD_INDEX


@pytest.mark.parametrize("rest", [True, False])
def test_lists_and_students_that_are_no_numbers(ctx, rest):
    x = logits_of(4, 300, BF16, 9)
    index, value = teacher(4, 300, 5, 10, x, 1.0)
    x[1, 17], value[2, 1] = NAN, NAN
    loss, saved, dx = new(4), new(4, 4), new(4, 300, dtype=BF16)
    ctx.distill_fwd(x, index, value, loss, rest=rest, saved=saved)
    ctx.distill_bwd(x, index, value, saved, torch.ones(4, device="cuda"), dx, rest=rest)
    bad = torch.tensor([False, True, True, False], device="cuda")
    assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(dx).any(1), bad)


def test_a_teacher_is_its_own_student(ctx):
    """The lists that token_logprobs writes are what distill reads: no divergence from oneself, at any temperature."""
    x = logits_of(50, 5003, F32, 11)
    for k, scale in ((1, 1.0), (20, 0.5), (128, 1.25)):
        top_lp, top_i = new(50, k), new(50, k, dtype=torch.int64)
        ctx.token_logprobs(x, scale=scale, top_logprob=top_lp, top_index=top_i)
        loss, saved, dx = new(50), new(50, 4), new(50, 5003)
        ctx.distill_fwd(x, top_i, top_lp, loss, rest=True, scale=scale, saved=saved)
        ctx.distill_bwd(x, top_i, top_lp, saved, torch.ones(50, device="cuda"), dx, rest=True, scale=scale)
        assert float(loss.abs().max()) < 2.0 ** -17 and float(dx.abs().max()) < 2.0 ** -17


def test_slope_of_the_forward_calls(ctx):
    """Differences of the calls themselves, FP32: step 2^-5, error 2^-12 of the slope's scale, rounding 2^-21 / 2^-5."""
    x = logits_of(5, 300, F32, 12)
    u = torch.randn((5, 300), device="cuda", generator=torch.Generator(device="cuda").manual_seed(13))
    t = torch.tensor([0, 5, 299, 7, 8], device="cuda")
    index, value = teacher(5, 300, 6, 14, x, 1.0)
    gl, gh = 1.0, 0.5

    def tokens(y):
        a, b, s = new(5), new(5), new(5, 4)
        ctx.token_logprobs(y, t, logprob=a, entropy=b, saved=s)
        return gl * a.double() + gh * b.double(), s

    def lists(y, rest):
        a, s = new(5), new(5, 4)
        ctx.distill_fwd(y, index, value, a, rest=rest, saved=s)
        return a.double(), s
    step, one = 2.0 ** -5, torch.ones(5, device="cuda")
    for f, back in ((tokens, lambda s, dx: ctx.token_logprobs_bwd(x, t, s, dx, g_logprob=gl * one, g_entropy=gh * one)),
                    (lambda y: lists(y, True), lambda s, dx: ctx.distill_bwd(x, index, value, s, one, dx, rest=True)),
                    (lambda y: lists(y, False), lambda s, dx: ctx.distill_bwd(x, index, value, s, one, dx, rest=False))):
        dx = new(5, 300)
        back(f(x)[1], dx)
        slope = (f(x + step * u)[0] - f(x - step * u)[0]) / (2 * step)
        want = (dx.double() * u.double()).sum(-1)
        assert float((slope - want).abs().max()) < 2.0 ** -7


def test_one_call_over_many_rows_is_many_calls(ctx):
    """A row's results do not depend on the other rows of its call, bit for bit; few rows may be spread over several SMs."""
    for vocab, dtype in ((32000, BF16), (5003, F32)):
        x = logits_of(700, vocab, dtype, 15)
        t = torch.arange(700, device="cuda") * 41 % vocab
        index, value = teacher(700, vocab, 16, 16, x, 1.0)

        def run(a, b):
            n = b - a
            o = [new(n) for _ in range(4)] + [new(n, 4), new(n, 9), new(n, 9, dtype=torch.int64), new(n, 4)]
            ctx.token_logprobs(x[a:b], t[a:b], logprob=o[0], entropy=o[1], lse=o[2], saved=o[4], top_logprob=o[5], top_index=o[6])
            ctx.distill_fwd(x[a:b], index[a:b], value[a:b], o[3], saved=o[7])
            d = [new(n, vocab, dtype=dtype) for _ in range(2)]
            ctx.token_logprobs_bwd(x[a:b], t[a:b], o[4], d[0], g_logprob=torch.ones(n, device="cuda"))
            ctx.distill_bwd(x[a:b], index[a:b], value[a:b], o[7], torch.ones(n, device="cuda"), d[1])
            return o + d
        whole = run(0, 700)
        again = run(0, 700)
        assert all(torch.equal(a, b) for a, b in zip(whole, again))
        for a, b in ((0, 1), (3, 40), (100, 300)):
            part = run(a, b)
            assert torch.equal(part[6], whole[6][a:b])
            for i in (0, 1, 2, 3, 5):
                torch.testing.assert_close(part[i], whole[i][a:b], rtol=2.0 ** -19, atol=2.0 ** -18)


def test_rows_far_apart(ctx):
    """Row distances that pass 32 bits."""
    ld, vocab = 1 << 29, 1003
    base = torch.empty(4 * ld + vocab, dtype=BF16, device="cuda")
    far = base.as_strided((5, vocab), (ld, 1))
    x = logits_of(5, vocab, BF16, 17)
    far.copy_(x)
    t = torch.arange(5, device="cuda")
    a, b, s, s2 = new(5), new(5), new(5, 4), new(5, 4)
    ctx.token_logprobs(far, t, logprob=a, saved=s)
    ctx.token_logprobs(x, t, logprob=b, saved=s2)
    assert torch.equal(a, b)
    dx = new(5, vocab, dtype=BF16)
    ctx.token_logprobs_bwd(x, t, s2, dx, g_logprob=torch.ones(5, device="cuda"))
    ctx.token_logprobs_bwd(far, t, s, far, g_logprob=torch.ones(5, device="cuda"))
    assert torch.equal(far, dx)


def test_graph_and_streams(ctx):
    x = logits_of(40, 5003, BF16, 18)
    index, value = teacher(40, 5003, 16, 19, x, 1.0)
    t = torch.arange(40, device="cuda")
    outs = [new(40), new(40), new(40, 4), new(40, 7), new(40, 7, dtype=torch.int64), new(40, 4), new(40, 5003, dtype=BF16), new(40, 5003, dtype=BF16), new(1)]
    one = torch.ones(40, device="cuda")

    def step():
        ctx.token_logprobs(x, t, logprob=outs[0], saved=outs[2], top_logprob=outs[3], top_index=outs[4])
        ctx.distill_fwd(x, index, value, outs[1], saved=outs[5])
        ctx.token_logprobs_bwd(x, t, outs[2], outs[6], g_logprob=one, d_amax=outs[8])
        ctx.distill_bwd(x, index, value, outs[5], one, outs[7], d_amax=outs[8])
    step()
    want = [o.clone() for o in outs]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for run in (step, graph.replay, step, graph.replay):
        for o in outs:
            o.view(torch.uint8).fill_(0x5A)
        run()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_neighbours_stay(ctx):
    for rows, vocab, k in ((3, 1003, 5), (1, 32000, 20), (4, 64, 64)):
        x = logits_of(rows, vocab, BF16, 20)
        index, value = teacher(rows, vocab, 8, 21, x, 1.0)
        t = torch.zeros(rows, dtype=torch.int64, device="cuda")
        flat = [new(rows + 32) for _ in range(4)] + [new(rows * k + 32), new(rows * k + 32, dtype=torch.int64), new(rows * 4 + 32), new(rows * 4 + 32)]
        size = [rows] * 4 + [rows * k] * 2 + [rows * 4] * 2
        grads = [new(rows + 2, vocab + 16, dtype=BF16) for _ in range(2)]
        before = [f.clone() for f in flat + grads]
        o = [f[16:16 + n] for f, n in zip(flat, size)]
        d = [f[1:rows + 1, 8:vocab + 8] for f in grads]
        ctx.token_logprobs(x, t, logprob=o[0], entropy=o[1], lse=o[2], saved=o[6].view(rows, 4), top_logprob=o[4].view(rows, k), top_index=o[5].view(rows, k))
        ctx.distill_fwd(x, index, value, o[3], saved=o[7].view(rows, 4))
        one = torch.ones(rows, device="cuda")
        ctx.token_logprobs_bwd(x, t, o[6].view(rows, 4), d[0], g_logprob=one)
        ctx.distill_bwd(x, index, value, o[7].view(rows, 4), one, d[1])
        for view, old, n in zip(o, before, size):
            view.copy_(old[16:16 + n])
        for view, old in zip(d, before[8:]):
            view.copy_(old[1:rows + 1, 8:vocab + 8])
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(flat + grads, before))


def test_largest_and_smallest_sizes(ctx, L):
    """The longest vocabulary of a list, more rows than a grid's second dimension has, one token."""
    x = logits_of(2, L.LOSS_VOCAB_MAX, F32, 22)
    index, value = teacher(2, L.LOSS_VOCAB_MAX, 256, 23, x, 1.0)
    index[1, :3] = torch.tensor([0, L.LOSS_VOCAB_MAX - 1, L.LOSS_VOCAB_MAX - 2], device="cuda")
    check_distill(ctx, x, index, value, True, 1.0, F32)
    check_tokens(ctx, x, torch.tensor([0, L.LOSS_VOCAB_MAX - 1], device="cuda"), 1.0, 128)
    for rows, vocab in ((70001, 7), (70001, 1)):
        x = logits_of(rows, vocab, BF16, 24)
        t = torch.arange(rows, device="cuda") % vocab
        saved, _ = check_tokens(ctx, x, t, 1.0, 1)
        dx, one = new(rows, vocab, dtype=BF16), torch.ones(1, device="cuda").expand(rows)
        ctx.token_logprobs_bwd(x, t, saved, dx, g_logprob=one)
        want = R.token_grad(x, t, one.double(), None, 1.0)
        torch.testing.assert_close(dx.double(), want, rtol=2.0 ** -7, atol=2.0 ** -19)


def test_calls_on_two_streams_at_once(ctx):
    """These calls have no workspace: two streams may make them on one context at the same time."""
    x = [logits_of(n, 32000, BF16, 25 + n) for n in (300, 40)]
    t = [torch.arange(n, device="cuda") for n in (300, 40)]
    lists = [teacher(n, 32000, 20, 26, a, 1.0) for n, a in zip((300, 40), x)]

    def run(i):
        n = x[i].shape[0]
        a, s, lp, ti, b, s2, d, amax = new(n), new(n, 4), new(n, 6), new(n, 6, dtype=torch.int64), new(n), new(n, 4), new(n, 32000, dtype=BF16), new(1)
        ctx.token_logprobs(x[i], t[i], logprob=a, saved=s, top_logprob=lp, top_index=ti)
        ctx.distill_fwd(x[i], *lists[i], b, saved=s2)
        ctx.distill_bwd(x[i], *lists[i], s2, torch.ones(n, device="cuda"), d, d_amax=amax)
        return a, s, lp, ti, b, s2, d, amax
    want = run(0), run(1)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [], []
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(run(i))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for r in got[i] for a, b in zip(r, want[i]))


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("vocab", [1003, 50257])
def test_padding_rows_may_hold_anything(ctx, vocab, rest):
    """A row whose list is padding has loss 0 and a gradient of zeros, whatever its logits are; in place too."""
    x = logits_of(4, vocab, BF16, 27)
    index, value = teacher(4, vocab, 5, 28, x, 1.0)
    index[1:3] = -1
    x[1], x[2, 17], value[1] = NAN, INF, NAN
    loss, saved, dx, amax = new(4), new(4, 4), new(4, vocab, dtype=BF16), new(1)
    ctx.distill_fwd(x, index, value, loss, rest=rest, saved=saved)
    ctx.distill_bwd(x, index, value, saved, torch.ones(4, device="cuda"), dx, rest=rest, d_amax=amax)
    assert loss[1:3].tolist() == [0.0, 0.0] and bool((dx[1:3] == 0).all()) and bool((dx[[0, 3]] != 0).any(1).all())
    assert float(amax) == float(dx.abs().max())
    ctx.distill_bwd(x, index, value, saved, torch.ones(4, device="cuda"), x, rest=rest)
    assert torch.equal(x, dx)


@pytest.mark.parametrize("rows,vocab,listed,dtype", [
    (1184, 1003, 20, BF16), (1183, 1003, 20, BF16), (2500, 1003, 64, F32), (2500, 1003, 65, F16), (1300, 515, 130, BF16), (1190, 131072, 7, BF16),
    (1190, 200003, 7, F16)])
def test_many_rows(ctx, rows, vocab, listed, dtype):
    """Both sides of each number of threads that a row may have: by rows, by listed tokens, by the list's shared memory."""
    x = logits_of(rows, vocab, dtype, 29)
    check_tokens(ctx, x, torch.arange(rows, device="cuda") * 7 % vocab, 1.0, 0, threads=64)
    index, value = teacher(rows, vocab, listed, 30, x, 1.0)
    for rest in (True, False):
        check_distill(ctx, x, index, value, rest, 1.0, dtype, threads=64, pick=slice(0, rows, 97))
