"""A decoder layer's self-attention over the paged FP8 cache, as a serving program runs it: prompts in chunks, then token by
token, sequences coming and going.  The linears have tests of their own; here every call's attention output is held to
the plain 64-bit implementation on the bytes that the cache holds at that moment, and the cached rows to the QKV
output that they were made from."""
import numpy as np
import pytest
import torch

import kv_reference as R
import oracle as O
from test_gpu_attn import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden,q_heads,kv_heads,head_dim,page", [(512, 8, 2, 64, 16), (256, 4, 4, 128, 32)])
def test_chunks_then_tokens(hidden, q_heads, kv_heads, head_dim, page):
    from paper_2309_17224_b200 import serving
    pool = serving.PagePool(24, page)
    cache = serving.empty_cache(24, kv_heads, page, head_dim)
    seen = {}

    def watch(q, k, batch):
        seen["q"], seen["k"] = q.double().cpu().numpy(), k.double().cpu().numpy()

    layer = serving.Fp8SelfAttention(hidden, q_heads, kv_heads, head_dim, cache, rotate=watch)
    attended = {}
    run = layer.ctx.attn_paged

    class Watched:
        def __getattr__(self, name):
            return getattr(serving.default_context(0), name)

        def attn_paged(self, cache, batch, q, out, causal=True):
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
            run(cache, batch, q, out, causal=causal, lse=lse)
            attended["out"], attended["lse"] = out.clone(), lse

    layer.ctx = Watched()
    g = torch.Generator(device="cuda").manual_seed(6)
    calls = [(["a", "b"], [70, 33]), (["a", "b", "c"], [40, 1, 20]), (["a", "b", "c"], [1, 1, 1]), (["c", "a"], [1, 1]),
             (["a", "b", "c"], [3, 2, 1])]
    for n, (seqs, new) in enumerate(calls):
        if n == 4:
            pool.release("b")          # a finished sequence leaves, another takes its name and its pages
        pool.extend(seqs, new)
        batch = pool.batch(seqs, new)
        x = torch.randn((sum(new), hidden), generator=g, device="cuda").to(torch.bfloat16)
        y = layer(x, batch)
        assert y.shape == (sum(new), hidden) and y.dtype == torch.bfloat16 and torch.isfinite(y).all()
        cpu = [t.cpu().numpy() for t in (cache.k8, cache.v8, cache.bk, cache.bv)]
        start, lens, rows = pool.indices(seqs, new)
        table = np.array(rows)
        want = R.attention(cpu, table, start, lens, seen["q"], head_dim ** -0.5, True, O.CONV_PAPER)
        check(attended["out"], attended["lse"], want, f"call {n}")
        for b in range(len(seqs)):
            kc, kb, _, _ = R.cached_rows(cpu, table, b, np.arange(lens[b] - new[b], lens[b]))
            for i in range(new[b]):
                for h in range(kv_heads):
                    codes, bias = R.quantise_row(seen["k"][start[b] + i, h], O.CONV_PAPER)
                    assert np.array_equal(kc[i, h], codes) and kb[i, h] == bias
        assert torch.equal(y, layer.out(attended["out"].flatten(1)))


def test_layer_refuses_another_cache():
    from paper_2309_17224_b200 import serving
    cache = serving.empty_cache(2, 2, 16, 64)
    with pytest.raises(ValueError):
        serving.Fp8SelfAttention(256, 4, 4, 64, cache)
