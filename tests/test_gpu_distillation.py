"""The distillation loss against 64 bits: vocabularies and lists of any size, rows without entries or labels, infinities, gradients."""
import math

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


def _case(rows, V, K, dtype, seed=0, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((rows, V), generator=g) * spread).to(dtype)
    t, ids = torch.topk(z.float() + torch.randn((rows, V), generator=g), min(K, V), dim=1)
    labels = torch.randint(-2, V + 2, (rows,), generator=g)
    return z.cuda(), t.to(dtype).cuda(), ids.cuda(), labels.cuda()


def _check(block, z, t, ids, labels, tau=1.0, w=0.0, what="", seed=5):
    leaf = z.detach().requires_grad_()
    loss = block.distillation_loss(leaf, t, ids, labels, temperature=tau, label_weight=w)
    g = torch.randn(loss.shape, generator=torch.Generator().manual_seed(seed)).cuda()
    dz, = torch.autograd.grad(loss, leaf, g)
    want = layers_oracle.distill(z, t, ids, labels, tau, w, g)
    assert loss.dtype == torch.float32 and dz.dtype == z.dtype
    assert_within(loss, *want["loss"], (what, "loss"))
    assert_within(dz, *want["dlogits"], (what, "dlogits"))
    with torch.no_grad():
        assert torch.equal(block.distillation_loss(z, t, ids, labels, temperature=tau, label_weight=w), loss)
    return loss, dz


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows, V, K", [(1, 1, 1), (1, 2, 1), (3, 7, 3), (5, 64, 8), (9, 65, 65), (4, 255, 1), (33, 1000, 100), (7, 2047, 5), (3, 2049, 300), (5, 4099, 64), (3, 32001, 128), (2, 50257, 513)])
def test_sizes(block, rows, V, K, dtype):
    z, t, ids, labels = _case(rows, V, K, dtype)
    for tau, w in ((1.0, 0.0), (2.0, 0.0), (1.0, 0.4), (3.0, 0.4), (0.5, 1.0), (2.0, 0.1)):
        _check(block, z, t, ids, labels, tau, w, (tau, w))
    _check(block, z, t, ids.int(), labels.int(), 2.0, 0.5, "int32")
    _check(block, z, t, ids, None, 2.0, 0.5, "no labels")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_lists_that_end_early(block, dtype):
    z, t, ids, labels = _case(12, 301, 40, dtype)
    n = torch.tensor([0, 1, 2, 39, 40, 0, 7, 13, 1, 0, 20, 40], device="cuda")
    past = torch.arange(40, device="cuda") >= n[:, None]
    by_id = ids.masked_fill(past, -1)
    want = _check(block, z, t, by_id, labels, 2.0, 0.3, "ids of -1")
    for other in (by_id.masked_fill(past, 301), by_id.masked_fill(past, 1 << 40), by_id.masked_fill(past, -(1 << 63))):
        for a, b in zip(_check(block, z, t.masked_fill(past, float("nan")), other, labels, 2.0, 0.3), want):
            assert torch.equal(a, b)
    for a, b in zip(_check(block, z, t.masked_fill(past, -math.inf), ids, labels, 2.0, 0.3, "logits of -infinity"), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_rows_with_nothing(block, dtype):
    """No entry and no label: zeros, whatever the logits are."""
    z, t, ids, labels = _case(6, 77, 9, dtype)
    z[1], z[2, 5], ids[1:4], labels[:] = float("nan"), float("inf"), -1, -100
    leaf = z.detach().requires_grad_()
    loss = block.distillation_loss(leaf, t, ids, labels, temperature=2.0, label_weight=0.5)
    dz, = torch.autograd.grad(loss.sum(), leaf)
    assert not loss[1:4].any() and not dz[1:4].any()
    keep = [0, 4, 5]
    want = layers_oracle.distill(z[keep], t[keep], ids[keep], labels[keep], 2.0, 0.5, torch.ones(3))
    assert_within(loss[keep], *want["loss"], "loss")
    assert_within(dz[keep], *want["dlogits"], "dlogits")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_the_same_place_twice(block, dtype):
    z, t, ids, labels = _case(7, 120, 30, dtype)
    ids[:, 5], ids[:, 6], ids[2] = ids[:, 4], ids[:, 4], 11
    labels = ids[:, 4].clone()          # (and the label's there too)
    labels[2] = 11
    _check(block, z, t, ids, labels, 2.0, 0.3)
    z, t, ids, labels = _case(3, 5000, 700, dtype)
    ids[:, 600:] = ids[:, :100]
    _check(block, z, t, ids, ids[:, 650], 1.0, 0.3)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_masked_vocabularies(block, dtype):
    """Logits of -infinity and of the type's lowest value: nothing there, no gradient."""
    for low in (-math.inf, torch.finfo(dtype).min):
        z, t, ids, labels = _case(5, 501, 20, dtype)
        for i in range(5):
            allowed = torch.zeros(501, dtype=torch.bool, device="cuda")
            allowed[ids[i]] = True
            allowed[labels[i].clamp(0, 500)] = True
            z[i] = torch.where(allowed, z[i], torch.tensor(low, dtype=dtype, device="cuda"))
        loss, dz = _check(block, z, t, ids, labels, 2.0, 0.3, low)
        assert not dz[z == low].any()
    # a place that the teacher names and the student rules out: infinitely far, with the gradient that there is
    z, t, ids, labels = _case(2, 501, 20, dtype)
    z[0, ids[0, 3]] = -math.inf
    leaf = z.detach().requires_grad_()
    loss = block.distillation_loss(leaf, t, ids)
    dz, = torch.autograd.grad(loss.sum(), leaf)
    p = torch.softmax(t[0].double(), 0)[3]
    assert loss[0] == math.inf and loss[1].isfinite() and abs(dz[0, ids[0, 3]].item() + p.item()) <= 2 * 2.0 ** -8 * p.item() and dz.isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_large_and_far_apart_logits(block, dtype):
    z, t, ids, labels = _case(6, 333, 20, dtype, spread=100.0)
    _check(block, z, t, ids, labels, 1.0, 0.3)
    _check(block, z, t, ids, labels, 0.01, 0.3)
    _check(block, z * 1e4, t * 1e4, ids, None, 1e3, 0.0)
    zero = torch.zeros(2, 64, dtype=dtype, device="cuda")
    loss, dz = _check(block, zero, zero[:, :4], torch.arange(4, device="cuda").expand(2, 4), None)
    assert_within(loss, torch.full((2,), math.log(16.0), dtype=torch.float64), torch.full((2,), 1e-6, dtype=torch.float64), "uniform")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_labels_alone(block, dtype):
    z, t, ids, labels = _case(40, 700, 1, dtype)
    none = t[:, :0], ids[:, :0]
    loss, dz = _check(block, z, *none, labels, 1.0, 1.0, "no list")
    again, _ = _check(block, z, t, ids, labels, 1.0, 1.0, "a list that does not weigh")
    assert torch.equal(loss, again)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strides_and_layouts(block, dtype):
    z, t, ids, labels = _case(12, 99, 10, dtype)
    wide = torch.full((12, 130), float("nan"), dtype=dtype, device="cuda")
    for first in (0, 1, 8, 31):
        wide.fill_(float("nan"))
        wide[:, first:first + 99] = z
        for a, b in zip(_check(block, wide[:, first:first + 99], t, ids, labels, 2.0, 0.3, first), _check(block, z, t, ids, labels, 2.0, 0.3)):
            # (a row that begins elsewhere in memory is summed by other lanes)
            assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if dtype == torch.bfloat16 else 1e-5, atol=1e-6)
    odd = z.flatten()[99:].view(11, 99)                 # (the first row itself off the boundary)
    _check(block, odd, t[1:], ids[1:], labels[1:], 2.0, 0.3, "odd")
    _check(block, z.view(3, 4, 99), t.view(3, 4, 10), ids.view(3, 4, 10), labels.view(3, 4), 2.0, 0.3, "three dimensions")
    _check(block, z.view(3, 4, 99)[:, 1:], t.view(3, 4, 10)[:, 1:], ids.view(3, 4, 10)[:, 1:], labels.view(3, 4)[:, 1:], 2.0, 0.3, "a part of the positions")
    _check(block, z[0], t[0], ids[0], labels[0], 2.0, 0.3, "one row")
    _check(block, z[:1].expand(5, 99), t[:5], ids[:5], labels[:5], 2.0, 0.3, "expanded")


def test_against_differences(block):
    z, t, ids, labels = _case(4, 37, 6, torch.float32)
    leaf = z.requires_grad_()
    g = torch.randn(4, generator=torch.Generator().manual_seed(1)).cuda()
    dz, = torch.autograd.grad(block.distillation_loss(leaf, t, ids, labels, temperature=2.0, label_weight=0.3), leaf, g)
    with torch.no_grad():
        for seed in range(4):
            v = torch.randn(z.shape, generator=torch.Generator().manual_seed(2 + seed)).cuda()
            h = 2.0 ** -7
            f = [(block.distillation_loss(z + k * h * v, t, ids, labels, temperature=2.0, label_weight=0.3).double() * g.double()).sum() for k in (1, -1)]
            slope, want = ((f[0] - f[1]) / (2 * h)).item(), (dz.double() * v.double()).sum().item()
            # the difference: h^2 / 6 of a third derivative of order ten, roundings of losses of order ten over 2 h
            assert abs(slope - want) < 1e-3


def test_mean_over_rows(block):
    """A gradient that is the same number for every row, as a mean's is."""
    z, t, ids, labels = _case(30, 257, 12, torch.bfloat16)
    leaf = z.detach().requires_grad_()
    block.distillation_loss(leaf, t, ids, temperature=2.0).mean().backward()
    assert_within(leaf.grad, *layers_oracle.distill(z, t, ids, None, 2.0, 0.0, torch.full((30,), 1 / 30))["dlogits"], "dlogits")


def test_refusals(block):
    z, t, ids, labels = _case(4, 50, 6, torch.float32)
    for args, kwargs, kind in (((z.cpu(), t, ids), {}, RuntimeError), ((z, t.cpu(), ids), {}, RuntimeError), ((z, t, ids.cpu()), {}, RuntimeError), ((z.half(), t.half(), ids), {}, TypeError),
                               ((z, t.bfloat16(), ids), {}, TypeError), ((z, t, ids.short()), {}, TypeError), ((z, t[:3], ids), {}, ValueError), ((z, t, ids[:, :3]), {}, ValueError),
                               ((z, t, ids, labels[:3]), {}, ValueError), ((z, t, ids, labels.float()), {}, TypeError), ((z, t, ids), {"temperature": 0.0}, ValueError),
                               ((z, t, ids), {"temperature": float("inf")}, ValueError), ((z, t, ids), {"temperature": float("nan")}, ValueError), ((z, t, ids), {"temperature": 1e-4}, RuntimeError),
                               ((z, t, ids), {"label_weight": 1.5}, ValueError), ((z, t, ids), {"label_weight": -0.1}, ValueError), ((z, t.clone().requires_grad_(), ids), {}, RuntimeError),
                               ((z[:, :0], t, ids), {}, ValueError)):
        with pytest.raises(kind):
            block.distillation_loss(*args, **kwargs)
    e = z[:0].clone().requires_grad_()
    loss = block.distillation_loss(e, t[:0], ids[:0])
    assert loss.shape == (0,) and torch.autograd.grad(loss.sum(), e)[0].shape == (0, 50)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("V, K", [(4099, 4099), (1000, 5000), (257, 256), (600, 255), (17, 1025)])
def test_long_lists(block, V, K, dtype):
    """Of a whole vocabulary, and longer than it: places many times over."""
    g = torch.Generator().manual_seed(3)
    z = (torch.randn((3, V), generator=g) * 2.5).to(dtype).cuda()
    ids = (torch.stack([torch.randperm(V, generator=g) for _ in range(3)]) if K == V else torch.randint(-3, V + 3, (3, K), generator=g)).cuda()
    t, labels = (torch.randn((3, K), generator=g) * 2).to(dtype).cuda(), torch.tensor([0, V - 1, -1]).cuda()
    for tau, w in ((1.0, 0.0), (2.0, 0.3)):
        _check(block, z, t, ids, labels, tau, w, (tau, w))
