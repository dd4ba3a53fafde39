"""The block operators while something watches: tracing, forward-mode tangents, hooks on what is saved.  As the sketched layers
(test_nn_native.py): the operators' Python functions serve these, and what they cannot do they refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _normal(seed, shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def _calls():
    """name -> (inputs, other inputs, call)"""
    from paper_2601_15473_amd import block
    w = _normal(1, (64,)), _normal(2, (64,))
    cos, sin, pos = torch.rand(40, 32, device="cuda"), torch.rand(40, 32, device="cuda"), torch.arange(17, device="cuda")
    ids = torch.randint(0, 50, (25,), generator=torch.Generator().manual_seed(3)).cuda()
    qkv = lambda seed: [_normal(seed + i, (2, 17, h, 64)) for i, h in enumerate((4, 2, 2))]  # noqa: E731
    heads = lambda seed: [_normal(seed, (17, 4, 64)), _normal(seed + 1, (17, 2, 64)), *w]  # noqa: E731
    return {
        "attention": (qkv(10), qkv(20), lambda q, k, v: block.attention(q, k, v, causal=True)),
        "head_norm_rope": (heads(10), heads(20), lambda q, k, a, b: block.head_norm_rope(q, k, a, b, cos, sin, pos)),
        "embedding": ([_normal(10, (50, 72))], [_normal(20, (50, 72))], lambda t: block.embedding(ids, t, 1.5)),
        "dropout": ([_normal(10, (9, 33))], [_normal(20, (9, 33))], lambda x: block.dropout(x, 0.3, 7, 5)),
        "dropout and residual": ([_normal(10, (9, 33)), _normal(11, (9, 33))], [_normal(20, (9, 33)), _normal(21, (9, 33))], lambda x, r: block.dropout(x, 0.3, 7, residual=r)),
    }


NAMES = ["attention", "head_norm_rope", "embedding", "dropout", "dropout and residual"]


def _tuple(y):
    return y if isinstance(y, tuple) else (y,)


@pytest.mark.parametrize("name", NAMES)
def test_tracing(name):
    """A trace makes the call again, on other inputs, with gradients or without."""
    inputs, other, call = _calls()[name]
    with torch.no_grad():
        traced = torch.jit.trace(call, tuple(inputs), check_trace=False)
        torch.full((1 << 20,), float("nan"), device="cuda")     # (what the allocator hands out next)
        for x in (inputs, other):
            for a, b in zip(_tuple(traced(*x)), _tuple(call(*x))):
                assert torch.equal(a, b)
    leaves = [[t.detach().clone().requires_grad_() for t in other] for _ in range(2)]
    got, want = _tuple(traced(*leaves[0])), _tuple(call(*leaves[1]))
    for a, b in zip(torch.autograd.grad(got, leaves[0], [t.detach() for t in got]), torch.autograd.grad(want, leaves[1], [t.detach() for t in want])):
        assert torch.equal(a, b)


def test_tracing_results_given():
    """head_norm_rope into tensors of the caller's."""
    from paper_2601_15473_amd import block
    (q, k, a, b), other, _ = _calls()["head_norm_rope"]
    cos, sin, pos = torch.rand(40, 32, device="cuda"), torch.rand(40, 32, device="cuda"), torch.arange(17, device="cuda")

    def call(q, k, a, b, oq, ok):
        return block.head_norm_rope(q, k, a, b, cos, sin, pos, out=(oq, ok))

    with torch.no_grad():
        traced = torch.jit.trace(call, (q, k, a, b, torch.empty_like(q), torch.empty_like(k)), check_trace=False)
        out = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        got = traced(*other, *out)
        for x, y, z in zip(got, out, block.head_norm_rope(*other, cos, sin, pos)):
            assert torch.equal(x, z) and torch.equal(y, z)


@pytest.mark.parametrize("requires_grad", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused(name, requires_grad):
    """No operator has a forward-mode derivative, and none drops a tangent without a word."""
    inputs, _, call = _calls()[name]
    for i in range(len(inputs)):
        with torch.autograd.forward_ad.dual_level():
            args = [t.detach().requires_grad_(requires_grad) for t in inputs]
            args[i] = torch.autograd.forward_ad.make_dual(args[i], torch.ones_like(args[i]))
            with pytest.raises(Exception, match="forward|jvp"):
                call(*args)


def test_tangents_are_refused_for_results_given():
    from paper_2601_15473_amd import block
    (q, k, a, b), _, _ = _calls()["head_norm_rope"]
    cos, sin, pos = torch.rand(40, 32, device="cuda"), torch.rand(40, 32, device="cuda"), torch.arange(17, device="cuda")
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(Exception, match="forward|jvp"):
            block.head_norm_rope(torch.autograd.forward_ad.make_dual(q, torch.ones_like(q)), k, a, b, cos, sin, pos, out=(torch.empty_like(q), torch.empty_like(k)))


@pytest.mark.parametrize("name", NAMES)
def test_transforms_are_refused(name):
    inputs, _, call = _calls()[name]
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda *a: call(*a))(*(torch.stack([t, t]) for t in inputs))


@pytest.mark.parametrize("name", NAMES)
def test_saved_tensors_hooks(name):
    inputs, _, call = _calls()[name]

    def step():
        leaves = [t.detach().requires_grad_() for t in inputs]
        out = _tuple(call(*leaves))
        return [*(o.detach() for o in out), *torch.autograd.grad(out, leaves, [o.detach() for o in out])]

    want = step()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
        got = step()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
