"""Layer norm against 64 bits, over the widths that its kernels are made for, with and without a residual, weights and gradients."""
import pytest
import torch

import layers_oracle
from block_oracle import assert_within

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _normal(seed, shape, dtype, scale=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + mean).to(dtype).cuda()


def _check(block, x, w, b, r, eps=1e-5, ds=True, what=""):
    leaves = {n: t.detach().requires_grad_() for n, t in (("x", x), ("weight", w), ("bias", b), ("residual", r)) if t is not None}
    out = block.layer_norm(x=leaves["x"], weight=leaves.get("weight"), bias=leaves.get("bias"), residual=leaves.get("residual"), eps=eps)
    y, s = out if r is not None else (out, None)
    dy = _normal(7, tuple(x.shape), x.dtype)
    dsum = _normal(8, tuple(x.shape), x.dtype) if r is not None and ds else None
    outs, grads = ([y, s], [dy, dsum]) if dsum is not None else ([y], [dy])
    got = dict(zip(leaves, torch.autograd.grad(outs, list(leaves.values()), grads)))
    want = layers_oracle.layer_norm(x, w, b, r, eps, dy, dsum)
    assert_within(y, *want["y"], (what, "y"))
    if r is not None:
        assert_within(s, *want["s"], (what, "s"))
        assert torch.equal(got["residual"], got["x"])
    assert_within(got["x"], *want["dx"], (what, "dx"))
    for n in ("weight", "bias"):
        if n in got:
            assert_within(got[n], *want["d" + n], (what, "d" + n))
    with torch.no_grad():
        again = block.layer_norm(x, w, b, r, eps=eps)
    for a, c in zip(again if r is not None else (again,), (y, s)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows, width", [(1, 8), (3, 24), (33, 64), (5, 72), (7, 128), (67, 256), (5, 264), (130, 512), (9, 520), (65, 768), (3, 1024), (4, 1032), (5, 2048),
                                         (1, 2056), (600, 4096), (2, 5000), (3, 6144), (2, 8192), (2, 8200), (1, 16384), (3, 16392), (2, 32768)])
def test_widths(block, rows, width, dtype):
    x, w, b, r = _normal(1, (rows, width), dtype, 1.0, 0.5), _normal(2, (width,), dtype, 0.3, 1.0), _normal(3, (width,), dtype, 0.3), _normal(4, (rows, width), dtype)
    _check(block, x, w, b, r, what="residual")
    _check(block, x, w, b, None, what="alone")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_what_may_be_missing(block, dtype):
    x, w, b, r = _normal(1, (2, 5, 96), dtype), _normal(2, (96,), dtype), _normal(3, (96,), dtype), _normal(4, (2, 5, 96), dtype)
    for weight in (w, None):
        for bias in (b, None):
            for residual in (r, None):
                for ds in (True, False):
                    _check(block, x, weight, bias, residual, ds=ds)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_gradient_of_the_sum_alone(block, dtype):
    x, r, w = (_normal(i, (9, 64), dtype).requires_grad_() for i in (1, 2, 3))
    w = w[0].detach().requires_grad_()
    y, s = block.layer_norm(x, w, None, r)
    ds = _normal(5, (9, 64), dtype)
    dx, dr, dw = torch.autograd.grad(s, (x, r, w), ds)
    assert torch.equal(dx, ds) and torch.equal(dr, ds) and not dw.any()


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_frozen_weights_and_inputs(block, dtype):
    x, w, b = _normal(1, (40, 256), dtype), _normal(2, (256,), dtype), _normal(3, (256,), dtype)
    dy = _normal(4, (40, 256), dtype)
    want = layers_oracle.layer_norm(x, w, b, dy=dy)
    for which in range(3):
        args = [t.detach().requires_grad_(i == which) for i, t in enumerate((x, w, b))]
        d, = torch.autograd.grad(block.layer_norm(*args), args[which], dy)
        assert_within(d, *want[("dx", "dweight", "dbias")[which]], which)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strided_rows_and_other_layouts(block, dtype):
    fused = _normal(1, (50, 3 * 128), dtype)
    x, r = fused[:, 128:256], fused[:, 256:]
    w, b = _normal(2, (128,), dtype), _normal(3, (128,), dtype)
    _check(block, x, w, b, r, what="slices")
    _check(block, fused[::2, :128], w, b, None, what="every other row")
    _check(block, _normal(4, (128, 50), dtype).t(), w, b, None, what="transposed")
    _check(block, _normal(4, (1, 128), dtype).expand(20, 128), w, b, r[:20], what="expanded")
    _check(block, _normal(5, (4, 6, 128), dtype).transpose(0, 1), w, b, None, what="three dimensions")
    _check(block, _normal(6, (50, 132), dtype)[:, 4:], w, b, None, what="off the boundary")
    _check(block, _normal(7, (128,), dtype), w, b, None, what="one row")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_a_mean_far_from_zero(block, dtype):
    """What is left behind the mean is what counts: the sums are about it."""
    x = _normal(1, (20, 512), torch.float32, 1.0, 1000.0 if dtype == torch.float32 else 30.0).to(dtype)
    _check(block, x, _normal(2, (512,), dtype), _normal(3, (512,), dtype), None)


def test_rows_of_one_value(block):
    """Nothing to divide by but eps: the bias."""
    for dtype in DTYPES:
        x, b = torch.full((3, 64), 0.25, dtype=dtype, device="cuda"), _normal(1, (64,), dtype)
        assert torch.equal(block.layer_norm(x, None, b), b.expand(3, 64))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_a_row_that_is_not_finite_is_its_own(block, dtype):
    x, w = _normal(1, (67, 256), dtype), _normal(2, (256,), dtype)
    bad = x.clone()
    bad[5, 3], bad[60] = float("nan"), float("inf")
    y, z = block.layer_norm(x, w), block.layer_norm(bad, w)
    assert z[5].isnan().all() and z[60].isnan().all()
    keep = torch.ones(67, dtype=torch.bool, device="cuda")
    keep[[5, 60]] = False
    assert torch.equal(y[keep], z[keep])


def test_against_differences(block):
    x, r, w, b = (_normal(i, s, torch.float32) for i, s in ((1, (6, 48)), (2, (6, 48)), (3, (48,)), (4, (48,))))
    dy, ds = _normal(5, (6, 48), torch.float32), _normal(6, (6, 48), torch.float32)
    leaves = [t.requires_grad_() for t in (x, w, b, r)]
    grads = torch.autograd.grad(block.layer_norm(*leaves, eps=1e-3), leaves, (dy, ds))
    value = lambda a: sum((o.double() * g.double()).sum() for o, g in zip(block.layer_norm(*a, eps=1e-3), (dy, ds)))  # noqa: E731
    with torch.no_grad():
        for i, g in enumerate(grads):
            for seed in range(3):
                v = _normal(20 + seed, tuple(g.shape), torch.float32)
                h = 2.0 ** -6
                moved = [[t + k * h * v if j == i else t for j, t in enumerate(leaves)] for k in (1, -1)]
                slope = ((value(moved[0]) - value(moved[1])) / (2 * h)).item()
                # the difference: h^2 of a third derivative of order one a value, and roundings of a sum of 600 over 2 h
                assert abs(slope - (g.double() * v.double()).sum().item()) < 0.02 * (g.double() * v.double()).abs().sum().item() + 1e-3


def test_refusals(block):
    x = torch.zeros(4, 64, device="cuda")
    for kwargs, kind in (({"x": x.cpu()}, RuntimeError), ({"x": x.half()}, TypeError), ({"x": x, "weight": x[0].bfloat16()}, TypeError),
                         ({"x": x, "weight": x[0].cpu()}, RuntimeError), ({"x": x, "weight": x[0, :32]}, ValueError), ({"x": x, "bias": x}, ValueError),
                         ({"x": x, "residual": x[:2]}, ValueError), ({"x": x[:, :12]}, RuntimeError), ({"x": x, "eps": -1.0}, RuntimeError),
                         ({"x": x, "eps": float("nan")}, RuntimeError), ({"x": torch.zeros(1, 32776, device="cuda")}, RuntimeError), ({"x": x[0, 0]}, ValueError)):
        with pytest.raises(kind):
            block.layer_norm(**kwargs)
    assert block.layer_norm(x[:0]).shape == (0, 64)
    e, w = x[:0].clone().requires_grad_(), x[0].clone().requires_grad_()
    dx, dw = torch.autograd.grad(block.layer_norm(e, w).sum(), (e, w))
    assert dx.shape == (0, 64) and not dw.any()
