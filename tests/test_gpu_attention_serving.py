"""Single tokens and pieces of a prompt on long caches, in both types: the forms that serve, at lengths past what a work-group takes at once."""
import pytest
import torch

import block_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape, lengths", [
    ((2, 1, 5000, 8, 1, 128), [5000, 4097]), ((3, 1, 9001, 4, 4, 64), [0, 9001, 8192]), ((1, 2, 12345, 16, 2, 80), None), ((2, 3, 6000, 5, 5, 24), [5999, 2]),
    ((1, 130, 7000, 4, 1, 128), [6913]),
], ids=str)
def test_long_caches(shape, lengths, dtype):
    from paper_2601_15473_amd import block
    B, Tq, Tk, H, Hkv, D = shape
    g = torch.Generator(device="cpu").manual_seed(Tk)
    q, kv = (torch.randn(s, generator=g).to(dtype).cuda() for s in ((B, Tq, H, D), (B, Tk, 2, Hkv, D)))
    k, v = kv[:, :, 0], kv[:, :, 1]
    kl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    value, bound = O.attention(q, k, v, None, lengths, True)["o"]
    O.assert_within(block.attention(q, k, v, k_lengths=kl, causal=True), value, bound, "o")
