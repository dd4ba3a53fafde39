"""Attention and its gradients against the plain form in 64 bits, where kernels go wrong: single tokens, odd lengths, rows that see
nothing, shared heads, strided views, whatever lies past the lengths."""
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


def _inputs(B, Tq, Tk, H, Hkv, D, dtype, seed=0):
    return (_normal(seed, (B, Tq, H, D), dtype, 1.5), _normal(seed + 1, (B, Tk, Hkv, D), dtype), _normal(seed + 2, (B, Tk, Hkv, D), dtype),
            _normal(seed + 3, (B, Tq, H, D), dtype))


def _poison():
    """Fills what the allocator hands out next with NaN: results have to be written in full."""
    for n in (1 << 12, 1 << 16, 1 << 20, 1 << 22):
        torch.full((n,), math.nan, device="cuda")


def _lengths(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def _check(block, q, k, v, do, ql=None, kl=None, causal=False, scale=None):
    want = O.attention(q, k, v, ql, kl, causal, scale, do)
    _poison()
    with torch.no_grad():
        o = block.attention(q, k, v, _lengths(ql), _lengths(kl), causal=causal, scale=scale)
    O.assert_within(o, *want["o"], "o of a forward pass alone")
    q, k, v = (t.detach().requires_grad_() for t in (q, k, v))
    o2 = block.attention(q, k, v, _lengths(ql), _lengths(kl), causal=causal, scale=scale)
    _poison()
    grads = torch.autograd.grad(o2, (q, k, v), do)
    O.assert_within(o2, *want["o"], "o")
    for name, g in zip(("dq", "dk", "dv"), grads):
        O.assert_within(g, *want[name], name)
    return o2.detach(), grads


SHAPES = [  # batch, q_len, k_len, heads, kv_heads, head_dim
    (1, 1, 1, 1, 1, 8), (2, 1, 7, 4, 2, 64), (1, 5, 3, 2, 1, 16), (2, 33, 33, 3, 1, 72), (1, 129, 257, 2, 2, 128),
    (3, 64, 64, 4, 4, 64), (1, 31, 300, 7, 1, 96), (1, 260, 131, 6, 2, 32), (2, 128, 128, 2, 1, 120), (1, 1, 1030, 16, 2, 128),
    (2, 3, 515, 8, 2, 80), (1, 515, 640, 2, 2, 64), (1, 300, 300, 5, 1, 40),
    (1, 70, 1500, 4, 2, 128), (2, 9, 2100, 12, 1, 64),   # ranges of the keys, over one tile of rows
    (1, 600, 330, 8, 1, 64), (2, 333, 260, 6, 2, 128),   # parts of the queries for few key heads
    (1, 1100, 1100, 8, 1, 64), (1, 1050, 1700, 16, 2, 104), (1, 3, 2100, 8, 4, 32),   # shares of the keys, for both directions or dq
    (2, 1100, 1100, 16, 8, 64), (3, 1030, 1090, 10, 5, 24), (1, 2100, 2100, 16, 16, 72), (1, 2060, 2060, 18, 18, 128),   # halves of a work-group
    (3, 200, 200, 8, 2, 64),   # parts of four tiles
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_plain_form(block, shape, causal, dtype):
    q, k, v, do = _inputs(*shape, dtype)
    _check(block, q, k, v, do, causal=causal)


RAGGED = [  # shape, queries', keys' lengths
    ((4, 40, 40, 2, 2, 64), [40, 0, 1, 33], [40, 0, 1, 33]),
    ((3, 70, 70, 4, 2, 128), None, [0, 70, 5]),
    ((3, 1, 200, 8, 2, 128), None, [0, 1, 200]),
    ((4, 2, 400, 8, 1, 64), None, [1, 2, 3, 400]),
    ((2, 150, 90, 2, 1, 48), [150, 20], [90, 64]),
    ((3, 130, 260, 3, 3, 64), [130, 128, -4], [260, 1000, 17]),   # out of range: clamped
    ((2, 257, 257, 2, 1, 128), [129, 257], [129, 256]),
    ((3, 520, 300, 8, 1, 64), [0, 520, 65], [300, 200, 3]),
    ((2, 1030, 1100, 8, 1, 64), [1030, 300], [1100, 700]),
    ((3, 1030, 1030, 4, 1, 128), [1030, 0, 64], [17, 1030, 961]),
    ((4, 1030, 1030, 8, 8, 64), [1030, 0, 64, 700], [1030, 1030, 65, 129]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("case", RAGGED, ids=lambda c: "x".join(map(str, c[0])))
def test_lengths_and_what_lies_past_them(block, case, causal, dtype):
    """NaN and infinities in rows that do not count reach nothing; rows that see nothing are zeros."""
    shape, ql, kl = case
    q, k, v, do = _inputs(*shape, dtype, seed=7)
    clean = [t.clone() for t in (q, k, v, do)]
    for b in range(shape[0]):
        n = shape[1] if ql is None else max(ql[b], 0)
        m = shape[2] if kl is None else max(kl[b], 0)
        q[b, n:], k[b, m:] = math.nan, math.nan
        v[b, m:], do[b, n:] = math.inf, -math.inf
    o, grads = _check(block, q, k, v, do, ql, kl, causal)
    o2, grads2 = _check(block, *clean, ql, kl, causal)
    for a, b in zip((o, *grads), (o2, *grads2)):
        assert torch.equal(a, b)


def test_rows_that_see_nothing(block):
    """More queries than keys under the causal mask: the first ones see none."""
    q, k, v, do = _inputs(1, 90, 20, 2, 1, 64, torch.bfloat16)
    o, (dq, _, _) = _check(block, q, k, v, do, causal=True)
    assert not o[:, :70].any() and not dq[:, :70].any() and o[:, 70:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_strided_views(block, dtype):
    """A fused projection's slices, heads before tokens, a cache with its own strides, a misaligned start, shared keys."""
    B, T, H, Hkv, D = 2, 70, 4, 2, 64
    fused = _normal(0, (B, T, H + 2 * Hkv, D), dtype)
    do = _normal(1, (B, T, H, D), dtype)
    _check(block, fused[:, :, :H], fused[:, :, H:H + Hkv], fused[:, :, H + Hkv:], do, causal=True)
    q = _normal(2, (B, H, T, D), dtype).transpose(1, 2)
    cache = _normal(3, (Hkv, 100, B, 2, D), dtype).permute(2, 1, 3, 0, 4)
    _check(block, q, cache[:, :T, 0], cache[:, :T, 1], do.transpose(1, 2).contiguous().transpose(1, 2))
    flat = _normal(4, (B * T * H * D + 1,), dtype)
    _check(block, flat[1:].view(B, T, H, D), fused[:, :, 4:6], fused[:, :, 6:], do)
    one = _normal(5, (B, T, 1, D), dtype)
    _check(block, q, one.expand(B, T, H, D), one.expand(B, T, H, D), do.sum(1, keepdim=True).expand(B, T, H, D))
    odd = _normal(6, (B, T, H, D + 1), dtype)[..., :D]
    _check(block, odd, odd[:, :, :2], odd[:, :, 2:], do)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [2, 40], ids=["few rows", "many"])
def test_scores_of_all_sizes(block, heads, dtype):
    """Scores that would overflow without the running maximum, rows with one key that takes all, equal scores, scales of either sign."""
    q, k, v, do = _inputs(1, 100, 200, heads, heads // 2, 64, dtype)
    _check(block, q * 40, k * 4, v, do)
    _check(block, q * 0, k, v, do, causal=True)
    _check(block, q, k, v, do, scale=-0.3)
    _check(block, q, k, v, do, scale=0.0)
    rising = (torch.linspace(0, 30, 200, device="cuda")[None, :, None, None] * torch.ones_like(k)).to(dtype)   # (every tile raises the maximum)
    _check(block, torch.ones_like(q), rising, v, do)


@pytest.mark.parametrize("heads", [1, 160], ids=["few rows", "many"])
def test_not_a_number_where_it_counts(block, heads):
    q, k, v, _ = _inputs(1, 40, 40, heads, heads, 64, torch.bfloat16)
    k[0, 17] = math.nan
    o = block.attention(q, k, v, causal=True)
    assert torch.isfinite(o[:, :17]).all() and torch.isnan(o[:, 17:]).all()


def test_runs_are_alike(block):
    q, k, v, do = (t.requires_grad_() for t in _inputs(2, 300, 300, 8, 2, 128, torch.bfloat16))
    first = None
    for _ in range(3):
        o = block.attention(q, k, v, causal=True)
        got = (o, *torch.autograd.grad(o, (q, k, v), do))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_gradients_against_differences(block):
    """<grad, d> against (f(x + e d) - f(x - e d)) / 2 e of the kernel's own results, e = 2^-5: off by the third derivative's e^2 / 6 and by 2^-22 / e of f's terms."""
    q, k, v, w = _inputs(1, 20, 30, 4, 2, 32, torch.float32)
    q, k, v = (t.requires_grad_() for t in (q, k, v))
    o = block.attention(q, k, v, causal=True)
    grads = torch.autograd.grad(o, (q, k, v), w)
    e = 2.0 ** -5
    f = lambda *t: (block.attention(*(x.detach() for x in t), causal=True).double() * w.double()).sum().item()  # noqa: E731
    for i in range(3):
        d = _normal(50 + i, tuple((q, k, v)[i].shape), torch.float32)
        d = d / d.norm()
        up, down = [q, k, v], [q, k, v]
        up[i], down[i] = (q, k, v)[i] + e * d, (q, k, v)[i] - e * d
        slope = (f(*up) - f(*down)) / (2 * e)
        assert abs(slope - (grads[i].double() * d.double()).sum().item()) <= 1e-3 * grads[i].double().norm().item() + 1e-4, i


def test_empty_tensors(block):
    q, k, v, _ = _inputs(2, 5, 6, 2, 1, 64, torch.bfloat16)
    assert block.attention(q[:, :0], k, v).shape == (2, 0, 2, 64)
    assert not block.attention(q, k[:, :0], v[:, :0]).any()
    assert block.attention(q[:0], k[:0], v[:0]).shape == (0, 5, 2, 64)
    q.requires_grad_()
    assert not torch.autograd.grad(block.attention(q, k[:, :0], v[:, :0]).sum(), q)[0].any()


def test_refusals(block):
    from paper_2601_15473_amd import libsk as sk
    q, k, v, _ = _inputs(2, 5, 6, 4, 2, 64, torch.bfloat16)
    with pytest.raises(ValueError):
        block.attention(q, k[:1], v[:1])
    with pytest.raises(ValueError):
        block.attention(q, k, v[:, :3])
    with pytest.raises(ValueError):
        block.attention(q[:, :, :3], k, v)
    with pytest.raises(TypeError):
        block.attention(q, k.float(), v)
    with pytest.raises(TypeError):
        block.attention(q.half(), k.half(), v.half())
    with pytest.raises(RuntimeError):
        block.attention(q, k.cpu(), v)
    with pytest.raises(ValueError):
        block.attention(q, k, v, k_lengths=torch.tensor([1], dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        block.attention(q, k, v, k_lengths=torch.tensor([1.0, 2.0], device="cuda"))
    for d in (60, 136):
        with pytest.raises(sk.SkError):
            block.attention(*(torch.zeros(1, 4, 2, d, device="cuda") for _ in range(3)))


def test_other_streams_and_integer_types(block):
    q, k, v, do = _inputs(2, 200, 200, 4, 2, 64, torch.bfloat16)
    want = block.attention(q, k, v, k_lengths=torch.tensor([200, 77], device="cuda"), causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(2048, 2048, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3                      # work in front of it on the stream
        q2 = q * 1                                      # made on the stream, right before
        got = block.attention(q2, k, v, k_lengths=_lengths([200, 77]), causal=True)
    side.synchronize()
    assert torch.equal(got, want)


def test_replays_from_a_graph(block):
    q, k, v, do = _inputs(2, 150, 150, 4, 2, 128, torch.bfloat16)
    cache_q = _normal(9, (2, 1, 4, 128), torch.bfloat16)
    lengths = _lengths([150, 30])
    eager = []

    def step():
        a, b, c = (t.detach().requires_grad_() for t in (q, k, v))
        o = block.attention(a, b, c, causal=True)
        return (o.detach(), *torch.autograd.grad(o, (a, b, c), do), block.attention(cache_q, k, v, k_lengths=lengths))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step()
    for rep in range(3):
        q.copy_(_normal(20 + rep, tuple(q.shape), torch.bfloat16, 1.5))
        lengths.copy_(torch.tensor([1 + 40 * rep, 150 - rep]))
        eager = step()
        for t in out:
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b), rep


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_offsets_past_32_bits(block, dtype):
    """A cache whose last keys lie more than 4 GB behind its first, and sequences that far apart, against dense copies of the same numbers."""
    tokens, apart = 700, 1 << 22 if dtype == torch.float32 else (1 << 22) - 8
    room = torch.zeros(tokens * apart, dtype=dtype, device="cuda")
    far = room.view(tokens, apart)[:, :2 * 64].view(1, tokens, 2, 64)
    far.copy_(_normal(0, (1, tokens, 2, 64), dtype))
    q, do = _normal(1, (1, 130, 4, 64), dtype), _normal(2, (1, 130, 4, 64), dtype)

    def both(k, v, q):
        a, b, c = (t.detach().requires_grad_() for t in (q, k, v))
        o = block.attention(a, b, c, causal=True)
        return (block.attention(q[:, :1], k, v), o.detach(), *torch.autograd.grad(o, (a, b, c), do))

    assert far.stride(1) * (tokens - 1) * far.element_size() > 1 << 32
    for x, y in zip(both(far, far, q), both(far.contiguous(), far.contiguous(), q)):
        assert torch.equal(x, y)
    batch = room[:(tokens * apart) // 64 // 256 * 64 * 256].view(2, -1)[:, :700 * 128].view(2, 700, 2, 64)      # two sequences half the room apart
    want = block.attention(q.expand(2, -1, -1, -1), batch.contiguous(), batch.contiguous())
    assert torch.equal(block.attention(q.expand(2, -1, -1, -1), batch, batch), want)


@pytest.mark.parametrize("shape", [(3, 50, 50, 4, 4, 64), (4, 100, 100, 4, 2, 128), (2, 700, 700, 6, 3, 32), (1, 2300, 2300, 4, 1, 32)], ids=lambda s: "x".join(map(str, s)))
def test_dq_of_few_keys_or_features_is_rounded_once(block, shape):
    """Rounding a value once is off by at most U of it, evenly spread: over all values by at most U / sqrt(3).  A second rounding on the way makes that
    1.4 times as much (0.0024 of rounding to bf16, where this is 0.00226 and one rounding 0.0017)."""
    q, k, v, do = _inputs(*shape, torch.bfloat16, seed=3)
    want = O.attention(q, k, v, None, None, True, None, do)["dq"][0]
    q.requires_grad_()
    dq, = torch.autograd.grad(block.attention(q, k, v, causal=True), q, do)
    assert (O.wide(dq) - want).norm() <= O.U[torch.bfloat16] / math.sqrt(3) * want.norm()
