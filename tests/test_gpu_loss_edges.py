"""Token log probabilities and distillation: one row through calls of different sizes.  Tolerances as in test_gpu_loss."""
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
