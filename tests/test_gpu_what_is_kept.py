"""What a stream keeps of its calls' scratch is bounded: a call that needs more takes it and gives it back."""
import time

import pytest
import torch

from paper_2601_15473_amd import nn as sknn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
def test_scratch_of_a_large_backward_pass(monkeypatch, native):
    from paper_2601_15473_amd import block
    from paper_2601_15473_amd import libsk as sk
    if not native:
        monkeypatch.setattr(block, "_native", None)
    g = torch.Generator(device="cpu").manual_seed(0)
    q, k, v = (torch.randn(s, generator=g).bfloat16().cuda().requires_grad_() for s in ((1, 8192, 8, 128), (1, 8192, 2, 128), (1, 8192, 2, 128)))
    shape = block._attention_shape(q, k, v, None, None, True, 0.1)
    assert sk.sk_attention_workspace_bytes(shape, 1) > 64 << 20
    sknn.release_workspaces()
    small = [t.detach()[:, :100].contiguous().requires_grad_() for t in (q, k, v)]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for inputs in (small, (q, k, v)):
        o = block.attention(*inputs, causal=True)
        grads = torch.autograd.grad(o, inputs, o.detach())
        del o, grads
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 64 << 20
    sknn.release_workspaces()
    for _ in range(200):      # (autograd's own thread lets go of a pass's gradients when it gets to it)
        if torch.cuda.memory_allocated() == before:
            break
        time.sleep(0.01)
    assert torch.cuda.memory_allocated() == before
