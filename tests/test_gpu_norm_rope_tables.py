"""The rotation's tables get no gradient, and a call that would want one is refused rather than left without."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("which", ["cos", "sin"])
@pytest.mark.parametrize("others", [False, True], ids=["tables alone", "heads too"])
def test_tables_that_require_grad(monkeypatch, which, others, native):
    from paper_2601_15473_amd import block
    if not native:
        monkeypatch.setattr(block, "_native", None)
    g = torch.Generator(device="cpu").manual_seed(0)
    q, k, w = (torch.randn(s, generator=g).cuda().requires_grad_(others) for s in ((5, 2, 64), (5, 1, 64), (64,)))
    cos, sin = (torch.rand(9, 32, device="cuda").requires_grad_(which == n) for n in ("cos", "sin"))
    pos = torch.arange(5, device="cuda")
    with pytest.raises(RuntimeError, match=f"{which} gets no gradient"):
        block.head_norm_rope(q, k, w, w, cos, sin, pos)
    want = block.head_norm_rope(q, k, w, w, cos.detach(), sin.detach(), pos)
    with torch.no_grad():
        got = block.head_norm_rope(q, k, w, w, cos, sin, pos)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
