"""Attention of rows that overlap in memory: one token (whose stride says nothing) and tensors expanded over their tokens.  What a tile holds past
the last row that counts is then that row again, not zeros."""
import math

import pytest
import torch

import block_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _normal(seed, shape, dtype, std=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def _lengths(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def _check(block, q, k, v, do, ql=None, kl=None, causal=False):
    want = O.attention(q, k, v, ql, kl, causal, None, do)
    q, k, v = (t.detach().requires_grad_() for t in (q, k, v))
    o = block.attention(q, k, v, _lengths(ql), _lengths(kl), causal=causal)
    O.assert_within(o, *want["o"], "o")
    for name, g in zip(("dq", "dk", "dv"), torch.autograd.grad(o, (q, k, v), do)):
        O.assert_within(g, *want[name], name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("shape", [(2, 1, 70, 2, 2, 64), (3, 1, 300, 16, 2, 128), (1, 1, 1, 4, 1, 32)], ids=lambda s: "x".join(map(str, s)))
def test_one_query_of_large_scores(block, shape, causal, dtype):
    """Scores past 100: an exponential of one of them, unshifted, is infinite."""
    B, Tq, Tk, H, Hkv, D = shape
    q, k = _normal(0, (B, Tq, H, D), dtype, 60.0), _normal(1, (B, Tk, Hkv, D), dtype, 4.0)
    assert (O.wide(q).view(B, Hkv, -1, D) @ O.wide(k).permute(0, 2, 3, 1)).max() * D ** -0.5 > 90
    _check(block, q, k, _normal(2, k.shape, dtype), _normal(3, q.shape, dtype), causal=causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lengths", [None, [100, 37], [0, 64]], ids=str)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_a_query_expanded_over_tokens(block, causal, lengths, dtype):
    B, T, H, D = 2, 100, 4, 64
    q, k = _normal(0, (B, 1, H, D), dtype, 60.0).expand(B, T, H, D), _normal(1, (B, T, 2, D), dtype, 4.0)
    _check(block, q, k, _normal(2, k.shape, dtype), _normal(3, q.shape, dtype), lengths, lengths, causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("queries", [1, 300], ids=["few rows", "many"])
@pytest.mark.parametrize("tokens", [1, 70], ids=["one key", "expanded"])
def test_values_that_are_not_finite(block, tokens, queries, dtype):
    """An infinite value that every query sees gives infinity: nothing past the last key adds zero times it."""
    B, H, D = 2, 8 if queries == 1 else 80, 64
    q, k = _normal(0, (B, queries, H, D), dtype), _normal(1, (B, 1, H, D), dtype).expand(B, tokens, H, D)
    v = _normal(2, (B, 1, H, D), dtype)
    v[..., 3] = math.inf
    o = block.attention(q, k, v.expand(B, tokens, H, D))
    assert (o[..., 3] == math.inf).all() and torch.isfinite(o[..., :3]).all() and torch.isfinite(o[..., 4:]).all()
