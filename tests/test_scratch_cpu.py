"""Whose scratch buffers a stream keeps, without a GPU."""
import torch
from torch._subclasses.fake_tensor import FakeTensor, FakeTensorMode

from paper_2601_15473_amd import nn as sknn


def test_stand_ins_are_not_kept(monkeypatch):
    """A call on tensors without memory is refused; the next one on its stream gets a buffer that has some."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(sknn, "_workspaces", type(sknn._workspaces)())
    device = torch.device("cpu")
    with FakeTensorMode():
        assert isinstance(sknn._workspace(device, 0, 1000), FakeTensor)
    ws = sknn._workspace(device, 0, 500)
    assert type(ws) is torch.Tensor and ws.data_ptr() != 0 and sknn._workspace(device, 0, 400) is ws


def test_recorded_and_large_calls_have_their_own(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(sknn, "_workspaces", type(sknn._workspaces)())
    device = torch.device("cpu")
    ws = sknn._workspace(device, 0, 500)
    large = sknn._workspace(device, 0, sknn._MAX_KEPT + 1)
    assert large.numel() > sknn._MAX_KEPT and sknn._workspace(device, 0, 500) is ws
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert sknn._workspace(device, 0, 500) is not ws
