"""Token log probabilities and distillation: one row through calls of different sizes, lists beside masked tokens.  Tolerances as in
test_gpu_loss."""
import math

import pytest
import torch

import head_reference as R
from test_gpu_loss import BF16, F16, F32, U, log_error, logits_of, new, teacher

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2309_17224_b200 import fp8lin
    return fp8lin.Context(0)


def test_parts_of_a_call_have_its_sums_and_gradients(ctx):
    """What the forward calls leave for the backward ones agrees within the bound of a sum's order, however many rows a call
    has; from the same sums a row's gradients are the same bits."""
    rows = 700
    for vocab, dtype in ((32000, BF16), (5003, F32), (1003, F16)):
        x = logits_of(rows, vocab, dtype, 31)
        t = torch.arange(rows, device="cuda") * 41 % vocab
        index, value = teacher(rows, vocab, 16, 32, x, 1.0)
        g = torch.linspace(-1, 1, rows, device="cuda")

        def forward(a, b):
            s = [new(b - a, 4), new(b - a, 4)]
            ctx.token_logprobs(x[a:b], t[a:b], saved=s[0])
            ctx.distill_fwd(x[a:b], index[a:b], value[a:b], new(b - a), saved=s[1])
            return s

        def backward(a, b, s):
            d = [new(b - a, vocab, dtype=dtype) for _ in range(3)]
            ctx.token_logprobs_bwd(x[a:b], t[a:b], s[0][a:b], d[0], g_logprob=g[a:b], g_entropy=g[a:b])
            ctx.distill_bwd(x[a:b], index[a:b], value[a:b], s[1][a:b], g[a:b], d[1])
            ctx.distill_bwd(x[a:b], index[a:b], value[a:b], s[1][a:b], g[a:b], d[2], rest=False)
            return d
        whole = forward(0, rows)
        grads = backward(0, rows, whole)
        lp = R.log_softmax(x, 1.0)[0]
        err, size = log_error(lp, 1.0, 64), R.entropy(lp)
        for a, b in ((0, 1), (3, 40), (100, 300)):
            part = forward(a, b)
            for w, p in zip(whole, part):
                assert torch.equal(w[a:b, 0], p[:, 0])
                # (both are off by the bound; of the listed tokens left out, too: fewer terms of the same kind)
                assert bool(((w[a:b, 1] - p[:, 1]).abs() <= 2 * (err[a:b] + U * w[a:b, 1].abs())).all())
                assert bool(((w[a:b, 3] - p[:, 3]).abs() <= 2 * (2 * err[a:b] + 4 * U * w[a:b, 3].abs())).all())
            assert bool(((whole[0][a:b, 2] - part[0][:, 2]).abs() <= 2 * ((err + 8 * U) * (2 + 2 * size))[a:b]).all())
            assert all(torch.equal(w[a:b], p) for w, p in zip(grads, backward(a, b, whole)))


def far_distill(x, index, value, scale, gl):
    """Loss and gradient (for gl) with the rest as an outcome, lists without padding; the unlisted tokens' shares of their own
    sum come from their own differences: p of the rest may be nothing in any number format."""
    z = scale * x.double()
    listed = torch.zeros_like(z, dtype=torch.bool).scatter_(1, index, True)
    most = z.amax(-1, keepdim=True)
    lp = (z - most) - torch.logsumexp(z - most, -1, keepdim=True)
    own = torch.where(listed, torch.full_like(z, -math.inf), z)
    top = own.amax(-1, keepdim=True)
    share = torch.softmax(own - top, -1)
    ln_rest = (top - most) + torch.logsumexp(own - top, -1, keepdim=True) - torch.logsumexp(z - most, -1, keepdim=True)
    q = value.double().exp()
    left = (1.0 - q.sum(-1, keepdim=True)).clamp(min=0.0)
    loss = (q * (value.double() - lp.gather(1, index))).sum(-1) + (left * (left.log() - ln_rest)).squeeze(-1)
    total = q.sum(-1, keepdim=True) + left
    grad = (total * lp.exp() - left * share).masked_fill(listed, 0.0) + torch.where(listed, total * lp.exp(), torch.zeros_like(lp))
    grad = grad.scatter_add(1, index, -q)
    return loss, scale * gl.double().unsqueeze(1) * grad


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 70001), (3, 32000), (40, 1003), (400, 5003)])
def test_a_rest_far_below_the_listed_tokens(ctx, rows, vocab, dtype):
    """The student's unlisted tokens all carry a finite mask.  Their gradients are shares of what the list leaves, -g q_r p_j / p_r,
    whatever p_r is: 32 bits hold p_j / p_r although neither of both."""
    for mask in (-100.0, -1e4, -1e9, torch.finfo(dtype).min):
        if mask < torch.finfo(dtype).min:
            continue
        for scale, inplace in ((1.0, False), (0.5, True)):
            x = logits_of(rows, vocab, dtype, vocab + rows)
            index, value = teacher(rows, vocab, 16, 33, x, 1.0)
            far = (x.float() if mask > -2e4 else torch.zeros_like(x, dtype=F32)) + mask   # (with differences of their own, or equal)
            keep = torch.zeros_like(x, dtype=torch.bool).scatter_(1, index, True)
            x.copy_(torch.where(keep, x, far.clamp(min=torch.finfo(dtype).min).to(dtype)))
            loss, saved, g = new(rows), new(rows, 4), torch.linspace(-1, 1, rows, device="cuda") + 0.25
            ctx.distill_fwd(x, index, value, loss, scale=scale, saved=saved)
            want, grad = far_distill(x, index, value, scale, g)
            # (sums as in check_distill; the loss is mostly q_r times the distance, of which q_r has 2^-24 / q_r of error)
            left = 1.0 - value.double().exp().sum(-1)
            err = (vocab / 128 + 64) * 2.0 ** -22
            assert bool(((loss.double() - want).abs() <= want.abs() * 8 * U + 40 * err + 64 * U).all()), (mask, scale)
            dx, amax = x if inplace else new(rows, vocab, dtype=dtype), new(1)
            ctx.distill_bwd(x, index, value, saved, g, dx, scale=scale, d_amax=amax)
            size = scale * g.double().abs().unsqueeze(1)
            bound = grad.abs() * (R.HALF[dtype] + err + 2.0 ** -15) + R.TINY[dtype] + torch.where(keep, size * (err + 2.0 ** -20), torch.zeros_like(size))
            off = (dx.double() - grad).abs()
            assert bool((off <= bound).all()), (mask, scale, float((off / bound).max()), float(left.min()))
            assert float(amax) == float(dx.float().abs().max())
