"""Rows that do not count are zeros, also where what counts is not finite: results and gradients of queries past their length and of queries that see no
key, gradients of keys past theirs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [  # shape, queries', keys' lengths: by tiles, few rows in ranges, shares, halves, parts
    ((2, 40, 40, 2, 2, 64), [33, 17], [20, 37]), ((3, 1, 2100, 8, 1, 128), [1, 0, 1], [2100, 600, 0]), ((2, 3, 700, 4, 2, 32), [2, 3], [650, 1]),
    ((1, 1100, 1700, 8, 1, 64), [1070], [1030]), ((4, 1030, 1100, 8, 8, 64), [1030, 5, 900, 700], [1000, 1100, 65, 129]), ((3, 200, 200, 8, 2, 64), [200, 130, 1], [199, 100, 200]),
    ((2, 300, 300, 40, 40, 128), [290, 100], [100, 290]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
@pytest.mark.parametrize("bad", [math.nan, math.inf], ids=str)
@pytest.mark.parametrize("shape, ql, kl", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_rows_that_do_not_count(shape, ql, kl, bad, which, causal, dtype):
    from paper_2601_15473_amd import block
    B, Tq, Tk, H, Hkv, D = shape
    g = torch.Generator(device="cpu").manual_seed(3)
    t = {n: torch.randn(s, generator=g).to(dtype).cuda() for n, s in (("q", (B, Tq, H, D)), ("k", (B, Tk, Hkv, D)), ("v", (B, Tk, Hkv, D)), ("do", (B, Tq, H, D)))}
    for b in range(B):                     # every sequence's last row that counts, which stands beside those that do not
        n = (ql if which in ("q", "do") else kl)[b]
        if n > 0:
            t[which][b, n - 1, :, 5] = bad
    lengths = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (ql, kl)]
    leaves = [t[n].requires_grad_() for n in "qkv"]
    o = block.attention(*leaves, *lengths, causal=causal)
    with torch.no_grad():
        alone = block.attention(*leaves, *lengths, causal=causal)
    dq, dk, dv = torch.autograd.grad(o, leaves, t["do"])
    for b in range(B):
        n, m = ql[b], kl[b]
        first = Tq if m == 0 else max(0, n - m) if causal else 0     # queries before it see no key
        for name, x in (("o", o), ("o alone", alone), ("dq", dq)):
            assert not x[b, n:].any() and not x[b, :min(first, n)].any(), (name, b)
        for name, x in (("dk", dk), ("dv", dv)):
            assert not x[b, m:].any(), (name, b)
