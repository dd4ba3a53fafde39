"""A query that sees no key has no gradient and gives none, whatever the gradient that comes back for it (a norm's at zero, say, is not a number)."""
import math

import pytest
import torch

import block_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf], ids=str)
@pytest.mark.parametrize("shape, ql, kl", [
    ((1, 90, 20, 2, 1, 64), None, None), ((2, 300, 200, 4, 2, 128), [300, 130], [200, 65]), ((2, 33, 40, 3, 3, 24), [33, 30], [0, 17]), ((1, 2100, 1600, 8, 8, 64), None, None),
    ((1, 1100, 1700, 8, 1, 64), [1100], [1030]),
], ids=str)
def test_gradients_of_rows_that_see_nothing(shape, ql, kl, bad, dtype):
    from paper_2601_15473_amd import block
    B, Tq, Tk, H, Hkv, D = shape
    g = torch.Generator(device="cpu").manual_seed(5)
    q, k, v, do = ((torch.randn(s, generator=g)).to(dtype).cuda() for s in ((B, Tq, H, D), (B, Tk, Hkv, D), (B, Tk, Hkv, D), (B, Tq, H, D)))
    lengths = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (ql, kl)]
    clean = do.clone()
    for b in range(B):
        n, m = Tq if ql is None else ql[b], Tk if kl is None else kl[b]
        do[b, :max(n - m, 0)], clean[b, :max(n - m, 0)] = bad, 0.0
    want = O.attention(q, k, v, ql, kl, True, None, clean)
    q, k, v = (t.requires_grad_() for t in (q, k, v))
    o = block.attention(q, k, v, *lengths, causal=True)
    for name, got in zip(("dq", "dk", "dv"), torch.autograd.grad(o, (q, k, v), do)):
        O.assert_within(got, *want[name], name)
