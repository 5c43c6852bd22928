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
