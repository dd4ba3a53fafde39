"""Dense layers on every kernel that the plans take for them (tests/test_layers_plans_cpu.py holds the sizes to that): small whole numbers over a power of two, whose products and
sums are exact in fp32 in any order, so that each result has one right value."""
import pytest
import torch

import layers_oracle
from block_oracle import F, U

pytestmark = pytest.mark.gpu

# tokens, inputs, outputs
SIZES = [
    # few rows, 32 and 64 columns to a work-group, in one range and in several
    (3, 200, 264), (5, 136, 8872), (13, 72, 8712), (16, 264, 1032), (24, 200, 9992), (31, 328, 520), (56, 200, 9512), (61, 264, 136), (67, 72, 4168), (7, 3272, 72), (11, 3336, 80),
    (22, 3592, 136), (41, 3240, 200), (130, 3272, 72), (4, 72, 3272), (12, 136, 3200), (20, 264, 3144), (37, 520, 3256),
    # tiles, rings of tiles, and either in ranges
    (258, 72, 200), (520, 264, 264), (1042, 96, 3096), (1100, 72, 2056), (8067, 72, 464), (19520, 72, 136), (33000, 72, 8), (33000, 8, 72), (34190, 144, 24), (33606, 24, 168), (16443, 144, 16),
    (1580, 224, 5328), (1580, 5168, 232), (42161, 144, 400), (59546, 288, 136), (136, 16368, 40), (130, 1096, 1800), (22, 4328, 760), (1, 704, 8224), (2, 12120, 264), (1, 136, 11400), (155, 528, 6880),
    (228, 10936, 656), (141, 2840, 7160), (5392, 1304, 11944),
    (325, 3272, 1424), (1411, 2816, 1456), (284, 2024, 8), (11266, 4488, 8), (153, 3472, 1160), (458, 1104, 3376), (423, 4232, 2984), (259, 24, 1872), (16852, 8, 2848), (289, 680, 3648),
    (4650, 1240, 136), (4113, 5640, 304), (1420, 8, 80), (15343, 8, 4680), (1347, 8, 8), (2265, 5608, 8),
]
# ... in fp32
SIZES_F32 = [(1, 8, 8), (5, 448, 16), (130, 136, 264), (2709, 576, 4208), (546, 3328, 3624), (6975, 1088, 984), (3014, 7704, 328)]


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _whole(seed, shape, dtype, most, over=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randint(-most, most + 1, shape, generator=g, device="cuda", dtype=torch.float32) * over).to(dtype)


def _case(T, I, O, dtype, bias=True, residual=True):
    # (sums of I, O and T products of up to four units: far below 2^24 of them; z of size one)
    over = 2.0 ** -round((I.bit_length() + 1) / 2)
    return (_whole(1, (T, I), dtype, 2), _whole(2, (O, I), dtype, 2, over), _whole(3, (O,), dtype, 2, 0.25) if bias else None, _whole(4, (T, O), dtype, 2, 0.5) if residual else None,
            _whole(5, (T, O), dtype, 2))


def _run(block, x, w, b, r, dy, act):
    leaves = {n: t.detach().requires_grad_() for n, t in (("x", x), ("weight", w), ("bias", b), ("residual", r)) if t is not None}
    y = block.linear(leaves["x"], leaves["weight"], leaves.get("bias"), leaves.get("residual"), activation=act)
    return y.detach(), dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), dy)))


def _same(got, want, what):
    want = want.to(got.dtype)
    if not torch.equal(got, want):
        off = (got != want).nonzero()
        raise AssertionError(f"{what}: {len(off)} of {got.numel()} values, the first at {off[0].tolist()}: {got[tuple(off[0])].item()} for {want[tuple(off[0])].item()}")


def _exact(block, T, I, O, dtype):
    for act, bias, residual in ((None, True, True), (None, False, False), ("relu", True, False), ("relu", False, True)):
        x, w, b, r, dy = _case(T, I, O, dtype, bias, residual)
        y, grads = _run(block, x, w, b, r, dy, act)
        z = x.float() @ w.float().t() + (0.0 if b is None else b.float())
        dz = dy.float() * (z > 0) if act == "relu" else dy.float()
        what = (T, I, O, act, bias, residual)
        _same(y, (z.clamp(min=0) if act == "relu" else z) + (0.0 if r is None else r.float()), (what, "y"))
        _same(grads["x"], dz @ w.float(), (what, "dx"))
        _same(grads["weight"], dz.t() @ x.float(), (what, "dweight"))
        if bias:
            _same(grads["bias"], dz.sum(0), (what, "dbias"))
        if residual:
            _same(grads["residual"], dy, (what, "dresidual"))
        with torch.no_grad():
            _same(block.linear(x, w, b, r, activation=act), y, (what, "y without gradients"))


@pytest.mark.parametrize("T, I, O", SIZES)
def test_products_are_exact(block, T, I, O):
    _exact(block, T, I, O, torch.bfloat16)


@pytest.mark.parametrize("T, I, O", SIZES_F32)
def test_products_are_exact_f32(block, T, I, O):
    _exact(block, T, I, O, torch.float32)


def _within(got, want, bound, what):
    off = (got.double() - want).abs() > bound
    assert torch.isfinite(got).all() and not off.any(), (what, int(off.sum()), got[off][:3].tolist(), want[off][:3].tolist())


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T, I, O", SIZES)
def test_smooth_activations(block, T, I, O, act):
    """z is exact, its rounding to bf16 for the derivative known; dz is rounded once, as an operand of two products."""
    u = U[torch.bfloat16]
    x, w, b, r, dy = _case(T, I, O, torch.bfloat16)
    y, grads = _run(block, x, w, b, r, dy, act)
    z = (x.float() @ w.float().t() + b.float()).double()
    a, _, ea, _ = layers_oracle.activation(act, z, False)
    want = a + r.double()
    _within(y, want, ea + 2 * F * (a.abs() + r.double().abs()) + u * want.abs(), "y")
    with torch.no_grad():
        assert torch.equal(block.linear(x, w, b, r, activation=act), y)
    _, slope, _, eslope = layers_oracle.activation(act, z.to(torch.bfloat16).double(), False)
    g, X, W = dy.double(), x.double(), w.double()
    dz, edz = g * slope, g.abs() * eslope + F * (g * slope).abs()
    once = edz + u * dz.abs()
    dx, dw, db = dz @ W, dz.t() @ X, dz.sum(0)
    _within(grads["x"], dx, once @ W.abs() + (O + 2) * F * (dz.abs() @ W.abs()) + u * dx.abs(), "dx")
    _within(grads["weight"], dw, once.t() @ X.abs() + (T + 2) * F * (dz.abs().t() @ X.abs()) + u * dw.abs(), "dweight")
    _within(grads["bias"], db, edz.sum(0) + (T + 4) * F * dz.abs().sum(0) + u * db.abs(), "dbias")
    assert torch.equal(grads["residual"], dy)


# ... where an operand spans more than 2^31 bytes over the tokens that a tile walks: offsets move on with an origin
SIZES_FAR = [(66050, 16384, 816), (66050, 2048, 16384), (148770, 8200, 14344)]


@pytest.mark.parametrize("T, I, O", SIZES_FAR)
def test_weight_gradients_past_two_gigabytes(block, T, I, O):
    x, w, _, _, dy = _case(T, I, O, torch.bfloat16, False, False)
    w = w.requires_grad_()
    dw, = torch.autograd.grad(block.linear(x, w), w, dy)
    want = torch.zeros(O, I, device="cuda")
    for i in range(0, T, 8192):      # (whole numbers below 2^24: exact)
        want += dy[i:i + 8192].float().t() @ x[i:i + 8192].float()
    _same(dw, want, "dweight")
