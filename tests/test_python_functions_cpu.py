"""The Python autograd functions without a GPU, the library's calls replaced: the order in which threads get to them."""
import contextlib
import threading
import time

import pytest
import torch

from paper_2601_15473_amd import block
from paper_2601_15473_amd import libsk as sk
from paper_2601_15473_amd import nn as sknn


def _attention():
    q, k, v = (torch.randn(1, 8, 2, 64, requires_grad=True) for _ in range(3))
    return block.AttentionFunction.apply(q, k, v, None, None, False, 0.125, True)


def _norm_rope():
    q, k, a, b = (torch.randn(s, requires_grad=True) for s in ((4, 2, 64), (4, 1, 64), (64,), (64,)))
    return block.NormRopeFunction.apply(q, k, a, b, torch.rand(9, 32), torch.rand(9, 32), torch.arange(4), 1e-6, False)[0]


def _embedding():
    return block.EmbeddingFunction.apply(torch.arange(4), torch.randn(9, 64, requires_grad=True), 1.0)


def _linear():
    x, U, b = (torch.randn(s, requires_grad=True) for s in ((16, 32), (16, 48), (48,)))
    return sknn.SKLinearFunction.apply(x, torch.randn(32, 16), U, b, 1, 16)


def _two_sided():
    x, U1, U2, b = (torch.randn(s, requires_grad=True) for s in ((16, 32), (16, 48), (32, 16), (48,)))
    return sknn.SKLinearTwoSidedFunction.apply(x, torch.randn(32, 16), U1, U2, torch.randn(16, 48), b, 1, 16)


@pytest.mark.parametrize("make", [_attention, _norm_rope, _embedding, _linear, _two_sided], ids=lambda f: f.__name__.strip("_"))
def test_a_scratch_buffer_is_one_threads_until_its_kernels_are_queued(monkeypatch, make):
    """Four threads on one stream: from when a call has the stream's buffer to the library's return no other call has it."""
    inside, between = [], []

    def workspace(device, stream, nbytes):
        inside.append(threading.get_ident())
        return torch.empty(256, dtype=torch.uint8)

    def call(*args):     # (a call of the library lets other threads run)
        mine = threading.get_ident()
        time.sleep(0.005)
        between.append(inside[-1] == mine)
        return sk.SK_OK

    for module in (block, sknn):
        monkeypatch.setattr(module, "_workspace", workspace)
        monkeypatch.setattr(module, "_on", lambda device: contextlib.nullcontext())
        monkeypatch.setattr(module, "_stream", lambda device: 0)
    monkeypatch.setattr(sknn, "_check", lambda *a: None)
    for name in ("sk_attention_fwd", "sk_attention_bwd", "sk_norm_rope_bwd", "sk_embedding_bwd", "sk_linear_fwd", "sk_linear_bwd", "sk_linear_bwd_two_sided"):
        monkeypatch.setattr(sk, name, call)
    monkeypatch.setattr(sk, "sk_norm_rope_fwd", lambda *a: sk.SK_OK)
    monkeypatch.setattr(sk, "sk_embedding_fwd", lambda *a: sk.SK_OK)
    start = threading.Barrier(4)

    def work():
        start.wait()
        for _ in range(3):
            out = make()
            out.backward(torch.ones_like(out))

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(between) >= 12 and all(between), between
