"""Calls on tensors without memory (torch's fake ones) are refused, and calls behind them are none the worse."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2601_15473_amd import nn as sknn

pytestmark = pytest.mark.gpu


def test_refused_and_forgotten(monkeypatch):
    from paper_2601_15473_amd import block
    q = torch.randn(1, 700, 2, 64, device="cuda").bfloat16()
    layer = sknn.SKLinear(64, 64, 1, 16, dtype=torch.bfloat16, seed=1)
    x = torch.randn(32, 64, device="cuda").bfloat16()
    want, y = block.attention(q[:, :1], q, q), layer(x)
    sknn.release_workspaces()
    mode = FakeTensorMode(allow_non_fake_inputs=True)
    with mode:
        fake = [mode.from_tensor(t) for t in (q, x)]
        with pytest.raises(Exception):
            block.attention(fake[0][:, :1], fake[0], fake[0])
        with pytest.raises(Exception):
            layer(fake[1])
    for native in (True, False):
        if not native:
            monkeypatch.setattr(sknn, "_native", None)
            monkeypatch.setattr(block, "_native", None)
        assert torch.equal(block.attention(q[:, :1], q, q), want) and torch.equal(layer(x), y)
