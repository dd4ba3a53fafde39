"""Norms with eps = 0: heads that are not there (a wave's turn past the last) leave nothing in the weights' gradients."""
import pytest
import torch

import block_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", [(7, 2, 1, 64), (5, 3, 5, 128), (3, 1, 1, 24), (6, 4, 4, 128), (9, 3, 1, 200)], ids=lambda c: "x".join(map(str, c)))
def test_gradients_without_eps(case, dtype):
    from paper_2601_15473_amd import block
    T, H, Hkv, D = case
    g = torch.Generator(device="cpu").manual_seed(T)
    q, k, wq, wk, dq, dk = ((torch.randn(s, generator=g)).to(dtype).cuda() for s in ((T, H, D), (T, Hkv, D), (D,), (D,), (T, H, D), (T, Hkv, D)))
    angle = torch.rand(20, D // 8 * 4, generator=g)
    cos, sin, pos = angle.cos().cuda(), angle.sin().cuda(), torch.arange(T, device="cuda")
    leaves = [t.requires_grad_() for t in (q, k, wq, wk)]
    grads = torch.autograd.grad(block.head_norm_rope(*leaves, cos, sin, pos, eps=0.0), leaves, (dq, dk))
    for i, (x, w, dy) in enumerate(((q, wq, dq), (k, wk, dk))):
        _, dx, dw = O.norm_rope(x, w, cos, sin, pos, 0.0, False, dy)
        # (bounds as tests/test_gpu_norm_rope.py counts them)
        r = O.wide(x).square().mean(-1, keepdim=True).rsqrt()
        xr = (O.wide(x) * r).abs()
        top = O.wide(dy).abs().amax(-1, keepdim=True) * 2
        both = r * (top * O.wide(w).abs().max()) * (1 + xr * xr.mean(-1, keepdim=True))
        O.assert_within(grads[i], dx, O.U[dtype] * dx.abs() + (D + 24) * O.F * 2 * both, ("dx", i))
        dw = dw.sum((0, 1))
        O.assert_within(grads[2 + i], dw, O.U[dtype] * dw.abs() + (T * x.shape[1] + D + 24) * O.F * (top * xr).sum((0, 1)), ("dw", i))
