"""head_norm_rope into tensors of the caller's is a change in place of them, for autograd too."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _inputs():
    g = torch.Generator(device="cpu").manual_seed(0)
    q, k, w = (torch.randn(s, generator=g).cuda() for s in ((5, 2, 64), (5, 1, 64), (64,)))
    cos = torch.rand(9, 32, device="cuda")
    return (q, k, w, w, cos, cos, torch.arange(5, device="cuda"))


@pytest.mark.parametrize("which", [0, 1])
def test_who_has_saved_them_finds_out(which):
    from paper_2601_15473_amd import block
    args = _inputs()
    x = args[which].clone().requires_grad_()
    y = x.exp()                                  # (saves its result)
    out = [torch.empty_like(args[0]), torch.empty_like(args[1])]
    out[which] = y.detach()                      # (shares its memory and its count of changes)
    with torch.no_grad():
        block.head_norm_rope(*args, out=tuple(out))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_results_with_gradients_are_refused():
    from paper_2601_15473_amd import block
    args = _inputs()
    out = torch.empty_like(args[0]).requires_grad_() * 1, torch.empty_like(args[1])
    with pytest.raises(RuntimeError, match="without gradients"):
        block.head_norm_rope(*args, out=out)
    with torch.no_grad():
        assert torch.equal(block.head_norm_rope(*args, out=out)[0], block.head_norm_rope(*args)[0])


def test_in_inference_mode_and_expanded():
    from paper_2601_15473_amd import block
    from paper_2601_15473_amd import libsk as sk
    args = _inputs()
    want = block.head_norm_rope(*args)
    with torch.inference_mode():
        out = torch.empty_like(args[0]), torch.empty_like(args[1])
        block.head_norm_rope(*args, out=out)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    with pytest.raises(sk.SkError):
        block.head_norm_rope(*args, out=(torch.empty(1, 2, 64, device="cuda").expand(5, 2, 64), torch.empty_like(args[1])))
