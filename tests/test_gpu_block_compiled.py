"""The block operators inside torch.compile: the same results and gradients, with and without gradients wanted, and the example model's step."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _normal(seed, shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def _calls():
    from paper_2601_15473_amd import block
    cos, sin, pos = torch.rand(40, 32, device="cuda"), torch.rand(40, 32, device="cuda"), torch.arange(17, device="cuda")
    ids = torch.randint(0, 50, (25,), generator=torch.Generator().manual_seed(3)).cuda()
    lengths = torch.tensor([17, 5], device="cuda")
    qkv = [_normal(i, (2, 17, h, 64)) for i, h in enumerate((4, 2, 2))]
    heads = [_normal(3, (17, 4, 64)), _normal(4, (17, 2, 64)), _normal(1, (64,)), _normal(2, (64,))]
    x = [_normal(i, (9, 33)) for i in (5, 6)]
    return {
        "attention": (qkv, lambda q, k, v: block.attention(q, k, v, causal=True)),
        "attention of lengths": (qkv, lambda q, k, v: block.attention(q * 2, k, v, lengths, lengths, scale=0.2)),
        "head_norm_rope": (heads, lambda q, k, a, b: block.head_norm_rope(q, k, a, b, cos, sin, pos)),
        "embedding": ([_normal(7, (50, 72))], lambda t: block.embedding(ids, t, 1.5) + 1),
        "dropout": (x[:1], lambda x: block.dropout(x, 0.3, 7, 5)),
        "dropout and residual": (x, lambda x, r: block.dropout(x, 0.3, (1 << 63) + 7, residual=r)),
    }


@pytest.mark.parametrize("name", ["attention", "attention of lengths", "head_norm_rope", "embedding", "dropout", "dropout and residual"])
def test_compiled(name):
    inputs, call = _calls()[name]

    def step(f):
        leaves = [t.detach().requires_grad_() for t in inputs]
        out = f(*leaves)
        out = out if isinstance(out, tuple) else (out,)
        with torch.no_grad():
            alone = f(*inputs)
        return [*(o.detach() for o in out), *(alone if isinstance(alone, tuple) else (alone,)), *torch.autograd.grad(out, leaves, [o.detach() for o in out])]

    want = step(call)
    torch._dynamo.reset()
    for a, b in zip(step(torch.compile(call, backend="eager")), want):
        assert torch.equal(a, b)


def test_a_compiled_model():
    from paper_2601_15473_amd import decoder
    model = decoder.Decoder(rows=40, width=128, layers=1, heads=2, kv_heads=1, head_dim=64, hidden=128, rank=64, p=0.1).train()
    ids = torch.randint(0, 40, (2, 17), generator=torch.Generator().manual_seed(1)).cuda()

    def step(f):
        model.zero_grad(set_to_none=True)
        y = f(ids)
        y.float().square().sum().backward()
        return [y.detach(), *(p.grad for p in model.parameters())]

    want = step(model)
    torch._dynamo.reset()
    for a, b in zip(step(torch.compile(model, backend="eager")), want):
        assert torch.equal(a, b)
