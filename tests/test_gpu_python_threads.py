"""The operators' Python functions (calls that the native ones leave) from threads on streams of their own and on one that they share: results as alone."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _normal(seed, shape):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).bfloat16().cuda()


def test_python_functions_of_threads(monkeypatch):
    from paper_2601_15473_amd import block
    monkeypatch.setattr(block, "_native", None)
    heads = [[_normal(9 * n + i, (1, n, h, 64)) for i, h in enumerate((8, 1, 1))] for n in (150, 700)]
    ids = torch.randint(0, 40, (900,), generator=torch.Generator().manual_seed(0)).cuda()
    table = _normal(5, (40, 64))
    w, cos, pos = _normal(6, (64,)), torch.rand(700, 32, device="cuda"), torch.arange(700, device="cuda")

    def once(i):
        x = [t.detach().requires_grad_() for t in heads[i % 2]]
        o = block.attention(*x, causal=True)
        t = table.detach().requires_grad_()
        y = block.embedding(ids[:100 + 400 * (i % 2)], t)
        q, a = heads[1][0][0].detach().requires_grad_(), w.detach().requires_grad_()
        n, _ = block.head_norm_rope(q, heads[1][1][0], a, w, cos, cos, pos)
        return [o.detach(), *torch.autograd.grad(o, x, o.detach()), *torch.autograd.grad(y, t, y.detach()), *torch.autograd.grad(n, (q, a), n.detach())]

    def work(stream, out, i):
        with torch.cuda.stream(stream):
            for _ in range(8):
                out[i] = once(i)
        stream.synchronize()

    want = [once(0), once(1)]
    torch.cuda.synchronize()
    for streams in ([torch.cuda.Stream() for _ in range(4)], [torch.cuda.Stream()] * 4):
        got = {}
        threads = [threading.Thread(target=work, args=(streams[i], got, i)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        for i in range(4):
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i % 2])), i
