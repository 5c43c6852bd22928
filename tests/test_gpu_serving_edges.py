"""The serving layer's odd calls: no rows, other types, contexts of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_step_in_which_no_sequence_has_new_tokens():
    from paper_2309_17224_b200 import serving
    pool = serving.PagePool(4, 16)
    layer = serving.Fp8SelfAttention(256, 4, 4, 64, serving.empty_cache(4, 4, 16, 64))
    pool.extend(["a"], [3])
    for seqs in (["a"], []):
        y = layer(torch.empty((0, 256), dtype=torch.bfloat16, device="cuda"), pool.batch(seqs, [0] * len(seqs)))
        assert y.shape == (0, 256) and y.dtype == torch.bfloat16


def test_layers_of_two_streams_have_contexts_of_their_own():
    """Prefill on one stream, decoding on another, at the same time: each gives the bits that it gives alone."""
    from paper_2309_17224_b200 import fp8lin, serving
    pool = serving.PagePool(80, 16)
    cache = serving.empty_cache(80, 2, 16, 64)
    own = fp8lin.Context(0)
    decode = serving.Fp8SelfAttention(256, 8, 2, 64, cache)
    prefill = serving.Fp8SelfAttention(256, 8, 2, 64, cache, ctx=own)
    assert prefill.ctx is own and prefill.qkv.ctx is own and prefill.out.ctx is own
    assert decode.ctx is serving.default_context(0) and decode.qkv.ctx is decode.ctx and decode.out.ctx is decode.ctx
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((300, 256), generator=g, device="cuda").to(torch.bfloat16)
    pool.extend(["a", "b"], [300, 600])
    decode(torch.randn((600, 256), generator=g, device="cuda").to(torch.bfloat16), pool.batch(["b"], [600]))
    whole, step = pool.batch(["a"], [300]), pool.batch(["b"], [1])
    want = prefill(x, whole), decode(x[:1], step)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [], []
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            got[0].append(prefill(x, whole))
        with torch.cuda.stream(streams[1]):
            got[1].append(decode(x[:1], step))
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(w, y) for y in many)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("tokens", [1, 200])
def test_inputs_of_other_types_give_the_same_bits(dtype, tokens):
    """Numbers that all three types hold: the same bytes after quantisation, so the same output and the same cache."""
    from paper_2309_17224_b200 import serving
    layer = serving.Fp8SelfAttention(256, 8, 2, 64, serving.empty_cache(16, 2, 16, 64))
    g = torch.Generator(device="cuda").manual_seed(10)
    x = torch.randint(-64, 65, (tokens, 256), generator=g, device="cuda").to(torch.bfloat16)
    pool = serving.PagePool(16, 16)
    pool.extend(["a"], [tokens])
    batch = pool.batch(["a"], [tokens])
    want, cache = layer(x, batch), layer.cache.k8.clone()
    got = layer(x.to(dtype), batch)
    assert got.dtype == torch.bfloat16 and torch.equal(got, want)
    pages = batch.page_table.flatten().long()
    assert torch.equal(layer.cache.k8[pages[:-1]], cache[pages[:-1]])
