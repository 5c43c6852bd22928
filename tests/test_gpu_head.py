"""The modules on the norm and loss calls: alone against 64-bit autograd, and together as a model's head uses them."""
import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def M():
    from paper_2309_17224_b200 import module
    return module


@pytest.fixture(scope="module")
def H():
    from paper_2309_17224_b200 import head
    return head


def randn(*shape, seed=0, dtype=BF16, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype,w_dtype", [(BF16, BF16), (BF16, F32), (F16, F32), (F32, F32)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("shape", [(3, 40, 512), (7, 1027), (1, 4096)])
def test_norm_module(M, kind, shape, dtype, w_dtype):
    n = shape[-1]
    norm = M.Norm(n, kind=kind, dtype=w_dtype)
    with torch.no_grad():
        norm.weight.copy_(1 + randn(n, seed=1, scale=0.2))
        if norm.bias is not None:
            norm.bias.copy_(randn(n, seed=2, scale=0.2))
    x, res, dy, dh = (randn(*shape, seed=s, dtype=dtype) for s in range(3, 7))
    xs, rs = x.clone().requires_grad_(True), res.clone().requires_grad_(True)
    y, h = norm(xs, rs)
    torch.autograd.backward((y, h), (dy, dh))
    want_h, want_y, _, _ = R.norm(x.view(-1, n), norm.weight.detach(), None if norm.bias is None else norm.bias.detach(), res.view(-1, n),
                                  layer=kind == "layer")
    dx, dw, db = R.norm_grad(dy.view(-1, n), want_h, norm.weight.detach(), dh.view(-1, n), layer=kind == "layer")
    assert torch.equal(h.view(-1, n), want_h)
    # a rounding of the type, and FP32 sums far below it; FP32: 2^-18 for sums of up to 4096 terms of size 1
    half = max(2 * R.HALF[dtype], 2.0 ** -18)
    for got, want in ((y, want_y), (xs.grad, dx)):
        torch.testing.assert_close(got.reshape(-1, n).double(), want, rtol=half, atol=half)
    half = max(2 * R.HALF[w_dtype], 2.0 ** -18)
    torch.testing.assert_close(norm.weight.grad.double(), dw, rtol=half, atol=half * 8)
    if db is not None and norm.bias is not None:
        torch.testing.assert_close(norm.bias.grad.double(), db, rtol=half, atol=half * 8)
    assert torch.equal(xs.grad, rs.grad) and xs.grad.data_ptr() != rs.grad.data_ptr()
    # inputs and gradients that are expanded numbers or rows
    row = x.reshape(-1, n)[:1].expand(5, n)
    a = row.detach().requires_grad_(True)
    z, h1 = norm(a, row)
    assert torch.equal(z[0], z[4]) and torch.equal(z[:1], norm(row[:1].clone(), row[:1].clone())[0])
    (z.sum() + h1.mean(0).sum()).backward()
    b = row.detach().clone().requires_grad_(True)
    z, h1 = norm(b, row.clone())
    torch.autograd.backward((z, h1), (torch.ones_like(z), torch.full_like(h1, 0.2)))
    torch.testing.assert_close(a.grad.float(), b.grad.float(), rtol=2.0 ** -6, atol=2.0 ** -6)   # (a fifth is no bf16 number)
    # without a residual, and with one of the two outputs unused
    xs.grad = None
    y1 = norm(xs)
    assert y1.shape == x.shape and torch.equal(y1, norm(x))
    _, h2 = norm(xs, rs)
    h2.backward(dh)
    assert torch.equal(xs.grad, dh)


@pytest.mark.parametrize("training", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind,tokens,K,N", [("layer", 300, 512, 272), ("rms", 40, 1040, 528), ("layer", 5, 4096, 1024), ("rms", 1, 8192, 256)])
def test_norm_linear_is_norm_then_linear(M, kind, tokens, K, N, dtype, training):
    """Bit for bit: outputs, sums, statistics of the cast, and every gradient."""
    fused = M.Fp8NormLinear(K, N, kind=kind, bias=True, dtype=dtype, margin=1)
    norm, linear = M.Norm(K, kind=kind, dtype=dtype), M.Fp8Linear(K, N, bias=True, dtype=dtype, margin=1)
    with torch.no_grad():
        fused.norm_weight.copy_(1 + randn(K, seed=11, scale=0.3))
        if kind == "layer":
            fused.norm_bias.copy_(randn(K, seed=12, scale=0.1))
            norm.bias.copy_(fused.norm_bias)
        norm.weight.copy_(fused.norm_weight)
        linear.weight.copy_(fused.weight)
        fused.bias.copy_(randn(N, seed=13, scale=0.1))
        linear.bias.copy_(fused.bias)
    fused.train(training)
    linear.train(training)
    for seed in (20, 30):                                          # (in eval() the second call finds the weight quantised)
        x, res = randn(tokens, K, seed=seed, dtype=dtype), randn(tokens, K, seed=seed + 1, dtype=dtype, scale=3.0)
        dy, dh = randn(tokens, N, seed=seed + 2, dtype=dtype, scale=1e-3), randn(tokens, K, seed=seed + 3, dtype=dtype, scale=1e-3)
        grads = []
        for which in (0, 1):
            a, b = x.clone().requires_grad_(True), res.clone().requires_grad_(True)
            for m in (fused, norm, linear):
                m.zero_grad()
            if which == 0:
                y, h = fused(a, b)
            else:
                n, h = norm(a, b)
                y = linear(n)
            if training:
                torch.autograd.backward((y, h), (dy, dh))
                grads.append([a.grad, b.grad] + ([fused.weight.grad, fused.bias.grad, fused.norm_weight.grad] if which == 0 else
                                                 [linear.weight.grad, linear.bias.grad, norm.weight.grad]) +
                             ([] if kind == "rms" else [(fused.norm_bias if which == 0 else norm.bias).grad]))
            grads.append([y, h])
        half = len(grads) // 2
        for one, two in zip(grads[:half], grads[half:]):
            assert all(torch.equal(p, q) for p, q in zip(one, two))
        assert torch.equal(fused.amax, linear.amax) and torch.equal(fused.bias_words, linear.bias_words)
        assert torch.equal(fused(x), linear(norm(x)))
    assert fused.ctx.device_flags() & 8 == 0


def test_norm_linear_with_constant_biases(M):
    const = (6, 4, 16)
    fused = M.Fp8NormLinear(512, 256, scaling="constant", constant_bias=const)
    norm, linear = M.Norm(512), M.Fp8Linear(512, 256, scaling="constant", constant_bias=const)
    with torch.no_grad():
        linear.weight.copy_(fused.weight)
    x = randn(70, 512, seed=1)
    a, b = x.clone().requires_grad_(True), x.clone().requires_grad_(True)
    y, z = fused(a), linear(norm(b))
    y.backward(randn(70, 256, seed=2, scale=1e-3))
    z.backward(randn(70, 256, seed=2, scale=1e-3))
    assert torch.equal(y, z) and torch.equal(a.grad, b.grad) and fused.bias_words.tolist() == list(const)


def test_refusals(M, H):
    with pytest.raises(ValueError):
        M.Fp8NormLinear(512, 256, scaling="predicted")
    with pytest.raises(ValueError):
        M.Norm(512, kind="batch")
    norm = M.Norm(512)
    x = randn(4, 512)
    for bad in ((x[:, :256], None), (x, x[:2]), (x, x.float())):
        with pytest.raises(ValueError):
            norm(*bad)
    logits, t = randn(4, 100), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call in (lambda: H.token_logprobs(logits, t[:3]), lambda: H.token_logprobs(logits, t.int()[:, None]), lambda: H.token_logprobs(logits, t.float()),
                 lambda: H.token_logprobs(logits, t, vocab=101), lambda: H.token_logprobs(logits, t, vocab=0),
                 lambda: H.distill_loss(logits, t[:3, None], torch.zeros(3, 1, device="cuda")),
                 lambda: H.distill_loss(logits, t[:, None], torch.zeros(4, 2, device="cuda"))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [None, 1003])
def test_losses_through_autograd(H, vocab, dtype):
    """Means and sums (gradients of one number for all rows), padded columns, a batch of two dimensions."""
    logits = randn(3, 21, 1008, seed=5, dtype=dtype, scale=2.0)
    columns = 1008 if vocab is None else vocab
    with torch.no_grad():
        logits[..., columns:] = float("nan")                       # not looked at
    t = torch.randint(0, columns, (3, 21), device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
    t[0, :4] = -1
    x = logits.clone().requires_grad_(True)
    lp, h = H.token_logprobs(x, t, scale=0.8, vocab=vocab)
    loss_scale = 256.0                                             # (FP16 gradients)
    (-lp.mean() * loss_scale + 0.1 * loss_scale * h.sum()).backward()
    flat = logits[..., :columns].reshape(-1, columns)
    n = 63
    want = R.token_grad(flat, t.view(-1), torch.full((n,), -loss_scale / n, device="cuda", dtype=torch.float64),
                        torch.full((n,), 0.1 * loss_scale, device="cuda", dtype=torch.float64), 0.8)
    got = x.grad.view(-1, 1008)
    assert bool((got[:, columns:] == 0).all())
    torch.testing.assert_close(got[:, :columns].double(), want, rtol=4 * R.HALF[dtype] + 2.0 ** -18, atol=2.0 ** -18 * loss_scale)
    value, index = H.top_tokens(logits + 0.5 * randn(3, 21, 1008, seed=7, dtype=dtype), 12, scale=0.8, vocab=vocab)
    for rest in (True, False):
        x.grad = None
        loss = H.distill_loss(x, index, value, scale=0.8, rest=rest, vocab=vocab)
        (loss * loss_scale).mean().backward()
        want_loss, grad = R.distill(flat, index.view(-1, 12), value.view(-1, 12), rest, 0.8)
        torch.testing.assert_close(loss.view(-1).double(), want_loss, rtol=2.0 ** -17, atol=2.0 ** -17)
        got = x.grad.view(-1, 1008)
        assert bool((got[:, columns:] == 0).all())
        torch.testing.assert_close(got[:, :columns].double(), grad * loss_scale / n, rtol=4 * R.HALF[dtype] + 2.0 ** -18, atol=2.0 ** -18 * loss_scale / n)


def make_head(H, hidden=512, vocab=1003):
    head = H.Fp8Head(hidden, vocab, kind="rms")
    with torch.no_grad():
        head.weight.copy_(randn(*head.weight.shape, seed=31, scale=0.05))
        head.norm_weight.copy_(1 + randn(hidden, seed=32, scale=0.2))
    return head


def test_a_student_learns_from_its_16_bit_self(H):
    """The run that the calls are for: a 16-bit teacher lists its most probable tokens, the FP8 head is distilled from them; the
    step's pieces by hand give the same bits."""
    head = make_head(H)
    x, res = randn(200, 512, seed=33), randn(200, 512, seed=34)
    h, n, _, _ = R.norm(x, head.norm_weight.detach(), None, res, layer=False)
    teacher = (n.float() @ head.weight.detach().float().t()).to(BF16)
    value, index = H.top_tokens(teacher, 24, vocab=head.vocab)
    a, b = x.clone().requires_grad_(True), res.clone().requires_grad_(True)
    loss = head.distill(a, index, value, residual=b)
    loss.mean().backward()
    assert loss.shape == (200,) and float(loss.detach().min()) > -2.0 ** -17
    got = [a.grad.clone(), b.grad.clone(), head.weight.grad.clone(), head.norm_weight.grad.clone()]
    assert bool((head.weight.grad[head.vocab:] == 0).all()) and bool(torch.isfinite(torch.cat([g.flatten().float() for g in got])).all())
    head.zero_grad()
    a, b = x.clone().requires_grad_(True), res.clone().requires_grad_(True)
    y, _ = head(a, b)
    want_loss, grad = R.distill(y.detach()[:, :head.vocab], index, value, True, 1.0)
    torch.testing.assert_close(loss.detach().double(), want_loss, rtol=2.0 ** -17, atol=2.0 ** -17)
    dlogits = torch.zeros_like(y)
    saved, out = torch.empty((200, 4), device="cuda"), torch.empty(200, device="cuda")
    head.ctx.distill_fwd(y.detach()[:, :head.vocab], index, value, out, saved=saved)
    head.ctx.distill_bwd(y.detach()[:, :head.vocab], index, value, saved, torch.full((1,), 1 / 200, device="cuda").expand(200), dlogits[:, :head.vocab])
    y.backward(dlogits)
    for g, w in zip(got, (a.grad, b.grad, head.weight.grad, head.norm_weight.grad)):
        assert torch.equal(g, w)
    # and the scores of given tokens from the same head
    t = index[:, 0].clone()
    lp, entropy = head.logprobs(x, t, residual=res)
    top, tokens = head.top(x, 3, residual=res)
    want, _ = R.log_softmax(y.detach()[:, :head.vocab], 1.0)
    torch.testing.assert_close(lp.detach().double(), want.gather(1, t[:, None]).squeeze(1), rtol=2.0 ** -18, atol=2.0 ** -18)
    torch.testing.assert_close(entropy.detach().double(), R.entropy(want), rtol=2.0 ** -16, atol=2.0 ** -16)
    assert torch.equal(tokens, R.top(y.detach()[:, :head.vocab], 3)) and top.shape == (200, 3)


def test_a_training_step_from_a_graph(H):
    """Forward and backward of the head captured and replayed, on inputs that change: the gradients of the eager step."""
    head = make_head(H)
    x, res = randn(160, 512, seed=35), randn(160, 512, seed=36)
    value, index = H.top_tokens(randn(160, 1008, seed=37, scale=3.0), 16, vocab=head.vocab)
    fixed = [t.clone() for t in (x, res, index, value)]
    params = list(head.parameters())

    def step():
        loss = head.distill(fixed[0], fixed[2], fixed[3], residual=fixed[1]).mean()
        return loss.detach(), torch.autograd.grad(loss, params)   # (no autograd graph outlives the step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = step()
    for seed in (40, 50):
        fixed[0].copy_(randn(160, 512, seed=seed))
        fixed[1].copy_(randn(160, 512, seed=seed + 1))
        graph.replay()
        replayed = [loss.clone()] + [g.clone() for g in grads]
        want, want_grads = step()
        assert torch.equal(replayed[0], want) and all(torch.equal(g, w) for g, w in zip(replayed[1:], want_grads))


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_self_attention_with_its_norm(M, norm):
    """A decoder layer's attention with the norm inside is the norm module and the layer without it, prompt and single tokens."""
    from paper_2309_17224_b200 import serving
    pools = [serving.PagePool(40, 16) for _ in range(2)]
    with_norm = serving.Fp8SelfAttention(512, 8, 2, 64, serving.empty_cache(40, 2, 16, 64), norm=norm)
    plain = serving.Fp8SelfAttention(512, 8, 2, 64, serving.empty_cache(40, 2, 16, 64))
    own = M.Norm(512, kind=norm, dtype=F32)
    with torch.no_grad():
        with_norm.qkv.norm_weight.copy_(1 + randn(512, seed=41, scale=0.2, dtype=F32))
        own.weight.copy_(with_norm.qkv.norm_weight)
        plain.qkv.weight.copy_(with_norm.qkv.weight)
        plain.out.weight.copy_(with_norm.out.weight)
        for new in ([150, 33], [1, 1], [1, 0]):
            batches = []
            for pool in pools:
                pool.extend(["a", "b"], new)
                batches.append(pool.batch(["a", "b"], new))
            x, res = randn(sum(new), 512, seed=42 + sum(new)), randn(sum(new), 512, seed=43 + sum(new))
            y, h = with_norm(x, batches[0], residual=res)
            n, want_h = own(x, res)
            assert torch.equal(h, want_h) and torch.equal(y, plain(n, batches[1]))
        y, h = with_norm(x[:0], batches[0])
        assert y.shape == (0, 512) and h.shape == (0, 512)
    with pytest.raises(ValueError):
        plain(x, batches[1], residual=res)
