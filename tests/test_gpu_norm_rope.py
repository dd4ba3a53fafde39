"""Norms of query and key heads with the rotation, and their gradients, against the plain form in 64 bits."""
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


def _tables(rows, rotary):
    a = torch.arange(rows)[:, None].double() * 10000.0 ** (-torch.arange(0, rotary, 2).double() / max(rotary, 1))
    return a.cos().float().cuda(), a.sin().float().cuda()


# One value is a product of five factors with two roundings each, one sum of D squares (half of whose error counts) and a sum of two
# products: D + 24 roundings of fp32 of the larger of the pair, and one of the storage type.  Gradients of x have a second sum.
def _bound(value, pair, dtype, D):
    return O.U[dtype] * value.abs() + (D + 24) * O.F * pair


CASES = [  # tokens, heads, kv_heads, head_dim, rotary, interleaved
    (1, 1, 1, 8, 8, False), (3, 2, 1, 16, 8, True), (5, 4, 2, 64, 64, False), (17, 3, 5, 72, 48, False), (130, 8, 2, 128, 128, True),
    (67, 5, 1, 80, 40, True), (9, 40, 8, 128, 128, False), (4, 2, 2, 256, 128, False), (33, 3, 0, 64, 64, False), (6, 2, 2, 96, 0, False),
    (5000, 2, 1, 32, 32, False), (300, 64, 8, 128, 64, False),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_against_the_plain_form(block, case, dtype):
    T, H, Hkv, D, rotary, interleaved = case
    qkv = _normal(T, (T, H + 2 * Hkv, D), dtype)
    q, k = qkv[:, :H], qkv[:, H:H + Hkv]                    # strided
    wq, wk = _normal(1, (D,), dtype), _normal(2, (D,), dtype)
    cos, sin = _tables(50, rotary)
    positions = torch.randint(-2, 54, (T,), generator=torch.Generator().manual_seed(T)).cuda()   # (clamped to 0 .. 49)
    dq, dk = _normal(3, (T, H, D), dtype), _normal(4, (T, Hkv, D), dtype)
    for pos in (positions, positions.int()):
        args = [t.detach().requires_grad_() for t in (q, k, wq, wk)]
        got = block.head_norm_rope(*args, cos, sin, pos, eps=1e-5, interleaved=interleaved)
        grads = torch.autograd.grad(got, args, (dq, dk))
        with torch.no_grad():
            again = block.head_norm_rope(q, k, wq, wk, cos, sin, pos, eps=1e-5, interleaved=interleaved)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
        for i, (x, w, dy) in enumerate(((q, wq, dq), (k, wk, dk))):
            if x.shape[1] == 0:
                assert got[i].shape == x.shape and not grads[2 + i].any()
                continue
            y, dx, dw = O.norm_rope(x, w, cos, sin, pos, 1e-5, interleaved, dy)
            r = (O.wide(x).square().mean(-1, keepdim=True) + 1e-5).rsqrt()
            size = (O.wide(x) * r * O.wide(w)).abs().amax(-1, keepdim=True) * 2
            O.assert_within(got[i], y, _bound(y, size, dtype, D), ("y", i))
            g = O.wide(dy).abs().amax(-1, keepdim=True) * 2 * O.wide(w).abs().max()
            xr = (O.wide(x) * r).abs()
            both = r * (g + xr * xr.mean(-1, keepdim=True) * g)
            O.assert_within(grads[i], dx, _bound(dx, 2 * both, dtype, D), ("dx", i))
            terms = O.wide(dy).abs().amax(-1, keepdim=True) * 2 * xr
            O.assert_within(grads[2 + i], dw.sum((0, 1)), O.U[dtype] * dw.sum((0, 1)).abs() + (T * x.shape[1] + D + 24) * O.F * terms.sum((0, 1)), ("dw", i))


def test_batches_and_results_in_place(block):
    B, S, H, Hkv, D = 3, 5, 4, 2, 64
    q, k = _normal(0, (B, S, H, D), torch.bfloat16), _normal(1, (B, S, Hkv, D), torch.bfloat16)
    wq, wk = _normal(2, (D,), torch.bfloat16), _normal(3, (D,), torch.bfloat16)
    cos, sin = _tables(40, D)
    pos = torch.arange(B * S, device="cuda").view(B, S)
    want = block.head_norm_rope(q, k, wq, wk, cos, sin, pos)
    flat = block.head_norm_rope(q.view(-1, H, D), k.view(-1, Hkv, D), wq, wk, cos, sin, pos.view(-1))
    assert torch.equal(want[0].view(-1, H, D), flat[0]) and torch.equal(want[1].view(-1, Hkv, D), flat[1])
    cache = torch.full((B * S, 2, Hkv, D), math.nan, dtype=torch.bfloat16, device="cuda")
    q2 = q.clone().view(-1, H, D)
    block.head_norm_rope(q2, k.view(-1, Hkv, D), wq, wk, cos, sin, pos.view(-1), out=(q2, cache[:, 1]))
    assert torch.equal(q2, flat[0]) and torch.equal(cache[:, 1], flat[1]) and torch.isnan(cache[:, 0]).all()


def test_heads_of_zeros(block):
    """The norm of a head of zeros is eps's alone."""
    z = torch.zeros(2, 3, 64, device="cuda").requires_grad_()
    w = torch.ones(64, device="cuda")
    cos, sin = _tables(4, 64)
    pos = torch.tensor([0, 3], device="cuda")
    q, k = block.head_norm_rope(z, z, w, w, cos, sin, pos, eps=1e-4)
    g, = torch.autograd.grad((q, k), z, (torch.ones_like(q), torch.zeros_like(k)))
    assert not q.any() and not k.any() and torch.isfinite(g).all() and g.abs().max() > 100


def test_gradients_against_differences(block):
    """As attention's: e = 2^-7 of a unit direction."""
    T, H, D = 6, 3, 64
    args = [_normal(0, (T, H, D), torch.float32), _normal(1, (T, 1, D), torch.float32), _normal(2, (D,), torch.float32), _normal(3, (D,), torch.float32)]
    args = [a.requires_grad_() for a in args]
    cos, sin = _tables(16, D)
    pos = torch.arange(T, device="cuda") + 7
    g = _normal(5, (T, H, D), torch.float32), _normal(6, (T, 1, D), torch.float32)
    grads = torch.autograd.grad(block.head_norm_rope(*args, cos, sin, pos), args, g)
    f = lambda a: sum((y.double() * w.double()).sum().item() for y, w in zip(block.head_norm_rope(*a, cos, sin, pos), g))  # noqa: E731
    e = 2.0 ** -7
    for i in range(4):
        d = _normal(10 + i, tuple(args[i].shape), torch.float32)
        d = d / d.norm()
        with torch.no_grad():
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + e * d, args[i] - e * d
            slope = (f(up) - f(down)) / (2 * e)
        assert abs(slope - (grads[i].double() * d.double()).sum().item()) <= 1e-3 * grads[i].double().norm().item() + 1e-3, i


def test_runs_are_alike(block):
    q, k = _normal(0, (3001, 8, 128), torch.bfloat16), _normal(1, (3001, 2, 128), torch.bfloat16)
    w = _normal(2, (128,), torch.bfloat16)
    args = [t.requires_grad_() for t in (q, k, w, w.clone())]
    cos, sin = _tables(3001, 128)
    pos = torch.arange(3001, device="cuda")
    runs = []
    for _ in range(2):
        y = block.head_norm_rope(*args, cos, sin, pos)
        runs.append((*y, *torch.autograd.grad(y, args, (q.detach(), k.detach()))))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_empty_and_refusals(block):
    from paper_2601_15473_amd import libsk as sk
    q, k, w = (torch.zeros(s, device="cuda") for s in ((4, 2, 64), (4, 1, 64), (64,)))
    cos, sin = _tables(8, 64)
    pos = torch.arange(4, device="cuda")
    assert block.head_norm_rope(q[:0], k[:0], w, w, cos, sin, pos[:0])[0].shape == (0, 2, 64)
    with pytest.raises(ValueError):
        block.head_norm_rope(q, k[:3], w, w, cos, sin, pos)
    with pytest.raises(ValueError):
        block.head_norm_rope(q, k, w[:32], w, cos, sin, pos)
    with pytest.raises(ValueError):
        block.head_norm_rope(q, k, w, w, cos, sin, pos[:3])
    with pytest.raises(ValueError):
        block.head_norm_rope(q, k, w, w, cos[:0], sin[:0], pos)
    with pytest.raises(TypeError):
        block.head_norm_rope(q, k, w.bfloat16(), w, cos, sin, pos)
    with pytest.raises(TypeError):
        block.head_norm_rope(q, k, w, w, cos.double(), sin.double(), pos)
    with pytest.raises(TypeError):
        block.head_norm_rope(q, k, w, w, cos, sin, pos.float())
    with pytest.raises(RuntimeError):
        block.head_norm_rope(q, k, w, w, cos.cpu(), sin, pos)
    with pytest.raises(RuntimeError):
        block.head_norm_rope(q.requires_grad_(), k, w, w, cos, sin, pos, out=(q.detach(), k))
    with pytest.raises(sk.SkError):
        block.head_norm_rope(*(t[..., :60].contiguous() for t in (q.detach(), k, w, w)), cos[:, :28].contiguous(), sin[:, :28].contiguous(), pos)
