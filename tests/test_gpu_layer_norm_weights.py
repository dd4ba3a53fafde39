"""The weight's gradient of a layer norm of a sum in bf16 is that of the sum before its rounding, over the widths of every kernel; against 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _normal(seed, shape, scale=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + mean).bfloat16().cuda()


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("mean", [0.0, 3.0])
@pytest.mark.parametrize("rows, width", [(1, 8), (67, 88), (33, 136), (9, 256), (130, 520), (40, 768), (21, 2056), (600, 4096), (5, 4104), (37, 8192), (50, 8200), (3, 16384), (35, 24584), (18, 32768)])
def test_of_the_sum_before_its_rounding(block, monkeypatch, rows, width, mean, native):
    if not native:
        monkeypatch.setattr(block, "_natively", lambda: False)
    x, r, w, dy = _normal(1, (rows, width), 0.5), _normal(2, (rows, width), 1.0, mean), _normal(3, (width,), 0.2, 1.0), _normal(4, (rows, width))
    for ds in (None, _normal(5, (rows, width))):
        w_, r_ = w.clone().requires_grad_(), r.clone().requires_grad_()
        y, s = block.layer_norm(x, w_, None, r_, eps=EPS)
        got, dr = torch.autograd.grad([y] if ds is None else [y, s], [w_, r_], [dy] if ds is None else [dy, ds])
        z, d = x.double() + r.double(), dy.double()
        mu = z.mean(-1, keepdim=True)
        inv = 1 / ((z - mu).square().mean(-1, keepdim=True) + EPS).sqrt()
        u = (z - mu) * inv
        want = (d * u).sum(0)
        # Half a step of the result; of each sum 2^-12 (four bits behind the eight: a 16th of a step, and a step is 2^-7 of the value at most, where a half has no ninth value; a
        # 32nd else, of which 2^-12 is all but the far end of a half); fp32: two roundings a term in u, the mean and deviation over the width, the products and the sum over rows
        e = 2.0 ** -23
        terms = (d.abs() * (z.abs() * (2.0 ** -11) + z.abs() * 2 * e + (z - mu).abs() * (8 + width ** 0.5) * e + mu.abs() * width ** 0.5 * e) * inv).sum(0) + rows ** 0.5 * 4 * e * (d * u).abs().sum(0)
        bound = want.abs() * 2.0 ** -8 * (1 + 2.0 ** -8) + terms
        assert ((got.double() - want).abs() <= bound).all(), (rows, width, ((got.double() - want).abs() - bound).max())
        if rows * width > 5000:   # ... and on the whole no further off than one rounding (2^-8 / sqrt 3 at most of a value, 0.0017 over the mantissas' lengths) and what 2^-12 a term leaves
            assert (got.double() - want).norm() / want.norm() < 0.0019
        assert dr.isfinite().all()


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_frozen_weights_keep_no_rest(block, monkeypatch, native):
    """Only the weight's gradient has use for it: beside bf16 tensors eight bytes a row are kept, and four bits a value."""
    if not native:
        monkeypatch.setattr(block, "_natively", lambda: False)
    x, r, w = _normal(1, (16, 64)), _normal(2, (16, 64)).requires_grad_(), _normal(3, (64,))
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.numel() * t.element_size() if t.dtype != torch.bfloat16 else 0) or t, lambda t: t):
        y, s = block.layer_norm(x, w, None, r)
        assert sum(kept) == 16 * 8
        kept.clear()
        y, s = block.layer_norm(x, w.requires_grad_(), None, r)
        assert sum(kept) == 16 * 8 + 16 * 64 // 2


def test_sums_that_are_not_finite(block):
    """Numbers past bf16's largest, infinities and NaN: a column's gradient is NaN or infinite where its sum is, and nowhere else if the row's dy is zero elsewhere."""
    x, r = torch.ones((8, 64)).bfloat16().cuda(), _normal(2, (8, 64))
    x[0, 3], x[1, 5], x[2, 7], r[2, 7] = float("inf"), float("nan"), 3.3e38, 3.3e38
    w = torch.ones(64).bfloat16().cuda().requires_grad_()
    y, s = block.layer_norm(x, w, None, r)
    dy = torch.zeros_like(y)
    dy[3:] = 1
    got, = torch.autograd.grad(y, w, dy)
    assert not s[:3].isfinite().all() and not y[:3].isfinite().all()
    z = x[3:].double() + r[3:].double()
    u = (z - z.mean(-1, keepdim=True)) / (z.var(-1, correction=0, keepdim=True) + EPS).sqrt()
    # (zeros times what is not finite are NaN, in torch's as here: only the finite rows' part is compared where the others have none)
    rows = torch.arange(3, 8)
    w2 = torch.ones(64).bfloat16().cuda().requires_grad_()
    y2, _ = block.layer_norm(x[rows], w2, None, r[rows])
    alone, = torch.autograd.grad(y2, w2, dy[rows])
    assert ((alone.double() - u.sum(0)).abs() <= u.sum(0).abs() * 2.0 ** -7 + u.abs().sum(0) * 2.0 ** -11).all()
    assert got.isnan().any()


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("width", [64, 2056, 8200])
def test_a_rest_of_what_is_not_finite(block, monkeypatch, width, native):
    """Rows that hold a NaN, an infinity or a sum past the largest number are NaN in their dx and in the sums over rows, as u is; every other row has the bits that it has without them."""
    if not native:
        monkeypatch.setattr(block, "_natively", lambda: False)
    x, r, w, dy = _normal(1, (9, width), 0.5), _normal(2, (9, width)), _normal(3, (width,), 0.2, 1.0), _normal(4, (9, width))
    x[7], r[7] = 1e15 * x[7], 1e15 * r[7]

    def call(x, r):
        w_, r_ = w.clone().requires_grad_(), r.clone().requires_grad_()
        y, s = block.layer_norm(x, w_, None, r_)
        return y.detach(), s.detach(), *torch.autograd.grad(y, [r_, w_], dy)

    y, s, dr, dw = call(x, r)
    assert y.isfinite().all() and dr.isfinite().all() and dw.isfinite().all()
    x2, r2 = x.clone(), r.clone()
    x2[0, 3], x2[4, 5], x2[5, 7], r2[5, 7] = float("inf"), float("nan"), 3.3e38, 3.3e38
    y2, s2, dr2, dw2 = call(x2, r2)
    bad = torch.tensor([0, 4, 5], device="cuda")
    good = torch.tensor([1, 2, 3, 6, 7, 8], device="cuda")
    assert y2[bad].isnan().all() and dr2[bad].isnan().all() and dw2.isnan().all()
    assert torch.equal(y2[good], y[good]) and torch.equal(s2[good], s[good]) and torch.equal(dr2[good], dr[good])
    assert s2[0, 3] == float("inf") and s2[4, 5].isnan() and s2[5, 7] == float("inf")
