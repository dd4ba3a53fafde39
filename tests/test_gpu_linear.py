"""Dense layers against 64 bits: every activation, sizes around the kernels' tiles, bias and residual or not, gradients."""
import pytest
import torch

import layers_oracle
from block_oracle import assert_within

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def _check(block, x, w, b, r, act, what=""):
    leaves = {n: t.detach().requires_grad_() for n, t in (("x", x), ("weight", w), ("bias", b), ("residual", r)) if t is not None}
    y = block.linear(leaves["x"], leaves["weight"], leaves.get("bias"), leaves.get("residual"), activation=act)
    dy = _normal(9, tuple(y.shape), x.dtype)
    got = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), dy)))
    want = layers_oracle.linear(x, w, b, r, act, dy)
    assert_within(y, *want["y"], (what, "y"))
    for n, d in got.items():
        assert_within(d, *want["d" + n], (what, "d" + n))
    with torch.no_grad():
        alone = block.linear(x, w, b, r, activation=act)
    assert_within(alone, *want["y"], (what, "y without gradients"))
    return y


def _case(T, I, O, dtype, bias=True, residual=True, seed=0):
    return (_normal(seed + 1, (T, I), dtype), _normal(seed + 2, (O, I), dtype, I ** -0.5), _normal(seed + 3, (O,), dtype, 0.5) if bias else None,
            _normal(seed + 4, (T, O), dtype) if residual else None)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("T, I, O", [(1, 8, 8), (1, 64, 40), (3, 8, 264), (8, 4096, 136), (17, 200, 328), (33, 72, 8), (64, 256, 256), (65, 264, 136), (127, 64, 128), (130, 1000, 72),
                                     (200, 96, 1032), (257, 512, 256), (300, 136, 520), (520, 264, 264), (1001, 128, 384)])
def test_sizes(block, T, I, O, dtype):
    for i, act in enumerate(ACTS):
        _check(block, *_case(T, I, O, dtype, bias=i % 2 == 0, residual=i % 3 != 1, seed=10 * i), act, what=act)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS, ids=str)
def test_bias_and_residual(block, act, dtype):
    for bias in (True, False):
        for residual in (True, False):
            _check(block, *_case(140, 192, 320, dtype, bias, residual), act, what=(bias, residual))


@pytest.mark.parametrize("act", [None, "gelu", "silu"], ids=str)
@pytest.mark.parametrize("T, I, O", [(2049, 512, 1536), (4097, 256, 2048), (1030, 2056, 1032), (8200, 136, 264), (700, 1032, 4104), (900, 1032, 1096), (2300, 1096, 1032), (6100, 1536, 1544), (9000, 200, 520)])
def test_large_tiles(block, T, I, O, act):
    """Sizes on the tiles of whole rounds, by every way through the plans."""
    _check(block, *_case(T, I, O, torch.bfloat16), act)


@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_over_their_range(block, act):
    """x the identity's rows: what comes out is the activation itself, from values that vanish to the largest there are."""
    for dtype in DTYPES:
        values = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 50.0, -50.0, 1e4, -1e4, 1e30, -1e30, 3e38, -3e38])])
        values = torch.cat([values, torch.zeros(-len(values) % 8)]).to(dtype).cuda()
        w = torch.zeros(len(values), 8, dtype=dtype, device="cuda")
        w[:, 0] = values
        x = torch.zeros(1, 8, dtype=dtype, device="cuda")
        x[0, 0] = 1.0
        b = torch.zeros(len(values), dtype=dtype, device="cuda").requires_grad_()
        y = block.linear(x, w, b, activation=act)
        slope, = torch.autograd.grad(y, b, torch.ones_like(y))
        z = values.double().cpu()
        a, s, ea, es = layers_oracle.activation(act, z.clamp(-1e5, 1e5), dtype == torch.float32)
        u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
        far = z.abs() > 1e3      # (a gate that is 0 or 1)
        a, s = torch.where(far, z.clamp(min=0), a), torch.where(far, (z > 0).double(), s)
        assert_within(y[0], a, torch.where(far, 0.0, ea) + (u + 4 * 2.0 ** -24) * a.abs(), (act, dtype), slack=1.1)
        if act == "relu":
            s = torch.where(z > 0, 1.0, 0.0)
        assert_within(slope, s, torch.where(far, 0.0, es) + (u + 4 * 2.0 ** -24) * s.abs(), (act, dtype, "slope"), slack=1.1)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strides_and_layouts(block, dtype):
    fused = _normal(1, (90, 3 * 64), dtype)
    w, b = _normal(2, (64, 64), dtype, 0.1), _normal(3, (64,), dtype)
    for act in (None, "gelu"):
        _check(block, fused[:, 64:128], w, b, fused[:, 128:], act, "slices")
        _check(block, fused[::3, :64], w, b, None, act, "every third row")
        _check(block, _normal(4, (1, 64), dtype).expand(70, 64), w, b, _normal(5, (1, 64), dtype).expand(70, 64), act, "expanded")
        _check(block, _normal(6, (64, 70), dtype).t(), w.t(), b, None, act, "transposed")
        _check(block, _normal(7, (2, 3, 5, 64), dtype), w, b, _normal(8, (2, 3, 5, 64), dtype), act, "four dimensions")
        _check(block, _normal(7, (64,), dtype), w, b, None, act, "one row")
        _check(block, _normal(8, (70, 68), dtype)[:, 4:], w, b[:64], None, act, "off the boundary")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_some_gradients(block, dtype):
    x, w, b, r = _case(140, 128, 192, dtype)
    dy = _normal(9, (140, 192), dtype)
    for act in (None, "silu"):
        want = layers_oracle.linear(x, w, b, r, act, dy)
        for which in range(1, 16):
            args = [t.detach().requires_grad_(bool(which >> i & 1)) for i, t in enumerate((x, w, b, r))]
            names = [n for i, n in enumerate(("dx", "dweight", "dbias", "dresidual")) if which >> i & 1]
            for n, d in zip(names, torch.autograd.grad(block.linear(*args, activation=act), [t for t in args if t.requires_grad], dy)):
                assert_within(d, *want[n], (act, which, n))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_rows_past_the_last_are_left_alone(block, dtype):
    """Through the C boundary, into the middle of buffers whose rest is to stay as it is; twice, with the same bits."""
    from paper_2601_15473_amd import libsk as sk
    for T, I, O in ((3, 64, 40), (130, 72, 136), (513, 264, 264)):
        x, w, b, r = _case(T, I, O, dtype)
        got = []
        for _ in range(2):
            room = torch.full((T + 4, O), 7.0, dtype=dtype, device="cuda")
            zroom = torch.full((T + 4, O), 7.0, dtype=dtype, device="cuda")
            s = sk.DenseShape(T, I, O, sk.SK_ACT_GELU, sk.SK_F32 if dtype == torch.float32 else sk.SK_BF16, I, O)
            n = max(sk.sk_dense_workspace_bytes(s, 0), sk.sk_dense_workspace_bytes(s, 1))
            ws = torch.full((max(n, 256) + 256,), 255, dtype=torch.uint8, device="cuda")      # (NaNs: nothing of it counts)
            sk.check(sk.sk_dense_fwd(s, x, w, b, r, room[2:], zroom[2:], ws, ws.numel(), torch.cuda.current_stream()))
            grads = [torch.full((k + 16,), 7.0, dtype=dtype, device="cuda") for k in (T * I, O * I, O)]
            sk.check(sk.sk_dense_bwd(s, x, w, zroom[2:], r, grads[0][8:], grads[1][8:], grads[2][8:], ws, n, torch.cuda.current_stream()))
            torch.cuda.synchronize()
            assert (ws[max(n, 256):] == 255).all()
            for t in (room, zroom):
                assert (t[:2] == 7).all() and (t[-2:] == 7).all()
            for g in grads:
                assert (g[:8] == 7).all() and (g[-8:] == 7).all()
            got.append([room, zroom, *grads])
        assert all(torch.equal(a, c) for a, c in zip(*got))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_a_row_that_is_not_finite_is_its_own(block, dtype):
    for T, I, O in ((5, 64, 64), (300, 136, 264)):
        x, w, b, r = _case(T, I, O, dtype)
        bad = x.clone()
        bad[T - 2] = float("nan")
        for act in ACTS:
            y, z = block.linear(x, w, b, r, activation=act), block.linear(bad, w, b, r, activation=act)
            assert z[T - 2].isnan().all(), act
            keep = torch.arange(T, device="cuda") != T - 2
            assert torch.equal(y[keep], z[keep]), act


def test_against_differences(block):
    for act in ("gelu", "gelu_tanh", "silu"):
        leaves = [t.requires_grad_() for t in _case(12, 24, 40, torch.float32)]
        dy = _normal(9, (12, 40), torch.float32)
        grads = torch.autograd.grad(block.linear(*leaves, activation=act), leaves, dy)
        with torch.no_grad():
            for i, g in enumerate(grads):
                v = _normal(20 + i, tuple(g.shape), torch.float32)
                h = 2.0 ** -7
                f = [(block.linear(*(t + k * h * v if j == i else t for j, t in enumerate(leaves)), activation=act).double() * dy.double()).sum() for k in (1, -1)]
                slope = ((f[0] - f[1]) / (2 * h)).item()
                terms = (g.double() * v.double())
                # the difference: h^2 / 6 of a third derivative of order one, and roundings of 480 values over 2 h
                assert abs(slope - terms.sum().item()) < 0.01 * terms.abs().sum().item() + 2e-3, (act, i)


def test_refusals(block):
    x, w = torch.zeros(4, 64, device="cuda"), torch.zeros(32, 64, device="cuda")
    for args, kwargs, kind in (((x.cpu(), w), {}, RuntimeError), ((x, w.cpu()), {}, RuntimeError), ((x.half(), w.half()), {}, TypeError), ((x, w.bfloat16()), {}, TypeError),
                               ((x, w.t()), {}, ValueError), ((x, w[0]), {}, ValueError), ((x, w, w[0]), {}, ValueError), ((x, w, None, x), {}, ValueError),
                               ((x, w), {"activation": "tanh"}, ValueError), ((x[:, :12], w[:, :12]), {}, RuntimeError), ((x, w[:12]), {}, RuntimeError)):
        with pytest.raises(kind):
            block.linear(*args, **kwargs)
    e, w = x[:0].clone().requires_grad_(), w.clone().requires_grad_()
    y = block.linear(e, w, activation="gelu")
    assert y.shape == (0, 32)
    dx, dw = torch.autograd.grad(y.sum(), (e, w))
    assert dx.shape == (0, 64) and not dw.any()
