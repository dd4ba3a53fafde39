"""Dropout: what is kept is the generator's, to the value, and the gradient draws it again."""
import math

import pytest
import torch

import block_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def test_generator_by_its_published_values():
    """Philox 4x32-10 of a counter and key of zeros, as its authors give it: 6627e8d5 e169c58d bc57ac4c 9b00dbd8."""
    assert O.words(8, 0, 0).tolist() == [0xe8d5, 0x6627, 0xc58d, 0xe169, 0xac4c, 0xbc57, 0xdbd8, 0x9b00]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 5003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999, 1.0, 1e-6])
def test_against_the_plain_form(block, n, p, dtype):
    seed, offset = 0xFEDCBA9876543210 + n, (1 << 40) + 17
    g = torch.Generator().manual_seed(n)
    x, r, dy = (torch.randn(n, generator=g).to(dtype).cuda() for _ in range(3))
    drop = round(p * 65536)
    kept = (O.words(n, seed, offset) >= drop).double() * (65536 / (65536 - drop) if drop < 65536 else 0.0)
    for residual in (None, r):
        x.requires_grad_()
        y = block.dropout(x, p, seed, offset, residual=residual)
        dx, = torch.autograd.grad(y, x, dy)
        base = 0.0 if residual is None else O.wide(residual)
        want = O.wide(x) * kept + base
        size = (O.wide(x) * kept).abs() + (0 if residual is None else base.abs())
        O.assert_within(y, want, O.U[dtype] * want.abs() + 3 * O.F * size, "y")
        O.assert_within(dx, O.wide(dy) * kept, (O.U[dtype] + 2 * O.F) * (O.wide(dy) * kept).abs(), "dx")


def test_many_values(block):
    """Past the first grid of threads the words go on; the share that is dropped is p's."""
    n = (1 << 25) + 3
    x = torch.ones(n, device="cuda")
    y = block.dropout(x, 0.1, 5, 6)
    zero = (y == 0).double().mean().item()
    assert abs(zero - 6554 / 65536) < 5 * math.sqrt(0.09 / n)
    for at in (0, n // 2 // 8 * 8, (n - 3) // 8 * 8):        # the counter of a piece in the middle, one at a time
        m = min(8, n - at)
        words = _piece(at // 8, 5, 6)[:m]
        assert torch.equal(y[at:at + m].cpu() != 0, words >= 6554)


def _piece(i, seed, offset):
    low, c, k = 0xFFFFFFFF, [i & 0xFFFFFFFF, i >> 32, offset, 0], [seed, 0]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return torch.tensor([w for v in c for w in (v & 0xFFFF, v >> 16)])


def test_offsets_and_seeds_differ(block):
    x = torch.ones(4096, device="cuda")
    masks = [block.dropout(x, 0.5, s, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0), (1 << 32, 0), (1, 1 << 32))]
    for i in range(len(masks)):
        for j in range(i):
            assert 0.45 < (masks[i] == masks[j]).double().mean().item() < 0.55


def test_dropped_values_and_strides(block):
    """What is dropped is gone whatever it was; any order and start of memory gives the same values at the same places."""
    x = torch.full((8192,), math.inf, device="cuda")
    y = block.dropout(x, 0.3, 11)
    assert set(y.unique().tolist()) == {0.0, math.inf}
    t = torch.randn(33, 64, device="cuda")
    want = block.dropout(t, 0.3, 11)
    assert torch.equal(block.dropout(t.t().contiguous().t(), 0.3, 11), want)
    flat = torch.zeros(33 * 64 + 1, device="cuda")
    flat[1:] = t.view(-1)
    assert torch.equal(block.dropout(flat[1:].view(33, 64), 0.3, 11), want)
    assert block.dropout(t[:0], 0.3, 11).shape == (0, 64)


def test_residual_gradient_and_second_derivative(block):
    x, r = (torch.randn(100, device="cuda", requires_grad=True) for _ in range(2))
    y = block.dropout(x, 0.4, 3, residual=r)
    dy = torch.randn(100, device="cuda", requires_grad=True)
    dx, dr = torch.autograd.grad(y, (x, r), dy, create_graph=True)
    assert torch.equal(dr, dy)
    back, = torch.autograd.grad(dx, dy, torch.ones_like(dx))
    assert torch.equal(back != 0, dx != 0)


def test_refusals(block):
    x = torch.zeros(8, device="cuda")
    for bad in (dict(p=-0.1, seed=1), dict(p=1.5, seed=1), dict(p=math.nan, seed=1), dict(p=0.5, seed=-1), dict(p=0.5, seed=1 << 64), dict(p=0.5, seed=1, offset=-1)):
        with pytest.raises(ValueError):
            block.dropout(x, **bad)
    with pytest.raises(ValueError):
        block.dropout(x, 0.5, 1, residual=x[:4])
    with pytest.raises(TypeError):
        block.dropout(x, 0.5, 1, residual=x.bfloat16())
    with pytest.raises(TypeError):
        block.dropout(x.half(), 0.5, 1)
    with pytest.raises(RuntimeError):
        block.dropout(x, 0.5, 1, residual=x.cpu())
