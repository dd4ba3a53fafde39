"""Layer norm, dense layers and the distillation loss where one tensor is two arguments, and where hooks give back what was saved in another layout."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def block():
    from paper_2601_15473_amd import block
    return block


def _normal(seed, shape, dtype):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def _tuple(y):
    return y if isinstance(y, tuple) else (y,)


def _gradients(out, leaves):
    return torch.autograd.grad(out, leaves, [torch.sin(torch.arange(o.numel(), device="cuda")).view(o.shape).to(o.dtype) for o in out])


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("name", ["residual of itself", "weight and bias", "layer's residual", "layer's weight", "layer's weight and residual"])
def test_one_tensor_as_two_arguments(block, monkeypatch, name, dtype, native):
    """The results are those of copies, and its gradient is the sum of theirs."""
    if not native:
        monkeypatch.setattr(block, "_natively", lambda: False)
    x, w, W = _normal(1, (72, 72), dtype), _normal(2, (72,), dtype), _normal(3, (72, 72), dtype)
    one, call = {
        "residual of itself": (x, lambda a, b: block.layer_norm(a, w, None, b)),
        "weight and bias": (w, lambda a, b: block.layer_norm(x, a, b)),
        "layer's residual": (x, lambda a, b: block.linear(a, W, None, b, activation="silu")),
        "layer's weight": (x, lambda a, b: block.linear(a, b, w, activation="gelu")),
        "layer's weight and residual": (W, lambda a, b: block.linear(x, a, w, b)),
    }[name]
    a, b, both = (one.clone().requires_grad_() for _ in range(3))
    want, got = _tuple(call(a, b)), _tuple(call(both, both))
    for u, v in zip(want, got):
        assert torch.equal(u, v)
    da, db = _gradients(want, [a, b])
    assert torch.equal(_gradients(got, [both])[0], da + db)


def _turned(t):
    """t's values with the first dimension's side by side, one element off a 16-byte boundary."""
    if t.dim() == 0 or t.numel() == 0:
        return t
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:]
    out = room.view(tuple(reversed(t.shape))).permute(*reversed(range(t.dim())))
    out.copy_(t)
    return out


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("name", ["layer norm", "layer norm and residual", "linear", "distillation"])
def test_hooks_that_change_the_layout(block, monkeypatch, name, dtype, native):
    if not native:
        monkeypatch.setattr(block, "_natively", lambda: False)
    x, w, W, r = _normal(1, (40, 72), dtype), _normal(2, (72,), dtype), _normal(3, (72, 72), dtype), _normal(4, (40, 72), dtype)
    g = torch.Generator(device="cpu").manual_seed(5)
    ids, labels = torch.stack([torch.randperm(72, generator=g)[:9] for _ in range(40)]).cuda(), torch.randint(72, (40,), generator=g).cuda()
    t = _normal(6, (40, 9), dtype)
    inputs, call = {
        "layer norm": ([x, w], lambda x, w: block.layer_norm(x, w)),
        "layer norm and residual": ([x, w, r], lambda x, w, r: block.layer_norm(x, w, None, r)),
        "linear": ([x, W, w, r], lambda x, W, w, r: block.linear(x, W, w, r, activation="gelu_tanh")),
        "distillation": ([x], lambda x: block.distillation_loss(x, t, ids, labels, temperature=2.0, label_weight=0.5)),
    }[name]
    leaves = [v.clone().requires_grad_() for v in inputs]
    want = _gradients(_tuple(call(*leaves)), leaves)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, _turned):
        out = _tuple(call(*leaves))
        got = _gradients(out, leaves)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
