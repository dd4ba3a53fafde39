"""What a backward pass with a graph of its own (create_graph) gives: gradients to use as any others, and a refusal where one is differentiated."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_gradients_with_a_graph(monkeypatch, native):
    from paper_2601_15473_amd import block
    if not native:
        monkeypatch.setattr(block, "_native", None)
    g = torch.Generator(device="cpu").manual_seed(0)
    q, k, v, do = (torch.randn(1, 12, 2, 64, generator=g).cuda() for _ in range(4))
    table, ids = torch.randn(9, 16, generator=g).cuda().requires_grad_(), torch.tensor([1, 1, 8], device="cuda")
    leaves = [t.requires_grad_() for t in (q, k, v)]
    plain = torch.autograd.grad(block.attention(*leaves, causal=True), leaves, do)
    graphed = torch.autograd.grad(block.attention(*leaves, causal=True), leaves, do.clone().requires_grad_(), create_graph=True)
    for a, b in zip(plain, graphed):
        assert not a.requires_grad and b.requires_grad and torch.equal(a, b)
    block.attention(*leaves, causal=True).backward(do, create_graph=True)          # (accumulated, changed in place, used in another loss)
    block.attention(*leaves, causal=True).backward(do)
    for t, a in zip(leaves, plain):
        assert torch.equal(t.grad, 2 * a)
        with torch.no_grad():
            t.grad.mul_(0.5)
        assert torch.equal(t.grad.detach(), a)
    dt, = torch.autograd.grad(block.embedding(ids, table).sum(), table, create_graph=True)
    for x in (graphed[0], graphed[2], dt):
        with pytest.raises(RuntimeError, match="libsk.*twice"):
            (x.square().sum() + q.sum()).backward()
