"""The example model of dense layers and layer norms, and a sketched one that learns from it: what they compute, from a cache too, and their gradients."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F = torch.nn.functional
SIZES = dict(rows=50, width=128, layers=2, heads=4, kv_heads=2, head_dim=32, hidden=192, context=64)


@pytest.fixture(scope="module")
def decoder():
    from paper_2601_15473_amd import decoder
    return decoder


def _ids(batch, n, seed=0):
    return torch.randint(0, 50, (batch, n), generator=torch.Generator().manual_seed(seed)).cuda()


def _rotated(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _reference(model, p, ids):
    """The model in 64 bits on the CPU, by torch's own operators; p: its parameters by name."""
    n, layer = ids.shape[1], model.layers[0]
    H, G, D = layer.heads, layer.kv_heads, layer.head_dim
    cos, sin = (t[:n].double().cpu()[:, None] for t in model.tables)
    x = p["table"][ids.cpu()] * model.scale
    for i in range(len(model.layers)):
        w = {k.split(".", 2)[2]: v for k, v in p.items() if k.startswith(f"layers.{i}.")}
        width = (x.shape[-1],)
        qkv = F.linear(F.layer_norm(x, width, w["norm_attention"], w["norm_attention_bias"]), w["qkv"], w["qkv_bias"]).unflatten(-1, (-1, D))
        q, k, v = qkv.split((H, G, G), 2)
        q, k = (_rotated(F.rms_norm(t, (D,), w[m], 1e-6), cos, sin) for t, m in ((q, "q_weight"), (k, "k_weight")))
        k, v = (t.repeat_interleave(H // G, 2) for t in (k, v))
        a = (q.transpose(1, 2) @ k.permute(0, 2, 3, 1)) * D ** -0.5
        a = a.masked_fill(torch.ones(n, n).triu(1) > 0, float("-inf")).softmax(-1)
        x = x + F.linear((a @ v.transpose(1, 2)).transpose(1, 2).flatten(2), w["out"], w["out_bias"])
        h = F.gelu(F.linear(F.layer_norm(x, width, w["norm_hidden"], w["norm_hidden_bias"]), w["up"], w["up_bias"]))
        x = x + F.linear(h, w["down"], w["down_bias"])
    return F.rms_norm(x, (x.shape[-1],), p["norm"], 1e-6) @ p["table"].t()


def test_dense_model(decoder):
    """Logits and every parameter's gradient; f32, 22 operators one behind the other, each off by at most some 200 terms' roundings (2^-24) of its size."""
    model = decoder.Decoder(**SIZES, dtype=torch.float32, p=0.0, dense=True).train()
    with torch.no_grad():
        for i, t in enumerate(model.parameters()):      # (biases that do something)
            t.add_(0.1 * torch.randn(t.shape, generator=torch.Generator().manual_seed(i)).to(t.dtype).cuda())
    ids = _ids(3, 21)
    out = model(ids)
    dy = torch.randn(out.shape, generator=torch.Generator().manual_seed(1)).cuda()
    grads = dict(zip(dict(model.named_parameters()), torch.autograd.grad(out, list(model.parameters()), dy)))
    wide = {n: t.detach().double().cpu().requires_grad_() for n, t in model.named_parameters()}
    want = _reference(model, wide, ids)
    tol = 2 * 22 * 200 * 2.0 ** -24
    assert (out.double().cpu() - want).norm() <= tol * want.norm()
    for n, g in zip(wide, torch.autograd.grad(want, list(wide.values()), dy.double().cpu())):
        assert (grads[n].double().cpu() - g).norm() <= tol * max(g.norm().item(), 1e-3), n


def test_cached_and_whole_passes_agree(decoder):
    model = decoder.Decoder(**SIZES, dtype=torch.float32, dense=True).eval()
    ids = _ids(3, 21)
    with torch.no_grad():
        whole = model(ids)
    cache = model.cache(3, 30)
    parts = [model.append(piece, cache) for piece in (ids[:, :9], ids[:, 9:10], ids[:, 10:18], *ids[:, 18:].split(1, 1))]
    assert torch.allclose(torch.cat(parts, 1), whole, rtol=1e-4, atol=1e-4 * whole.abs().max().item())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_dense_model_trains_and_teaches(decoder, dtype):
    """Both commands' steps run, with dropout; the teacher stays what it was."""
    teacher, student = decoder.Decoder(**SIZES, dtype=dtype, dense=True), decoder.Decoder(**SIZES, rank=64, dtype=dtype, seed=5)
    losses = []
    first = [t.detach().clone() for t in teacher.parameters()]
    decoder.train(teacher, 3, batch=4, half=8, report=lambda step, loss: losses.append(loss.item()))
    assert any(not torch.equal(a, b) for a, b in zip(first, teacher.parameters()))
    held = [t.detach().clone() for t in teacher.parameters()]
    begun = [t.detach().clone() for t in student.parameters()]
    decoder.distill(student, teacher, 3, batch=4, half=8, report=lambda step, loss: losses.append(loss.item()))
    assert all(torch.equal(a, b) for a, b in zip(held, teacher.parameters()))
    assert all(not torch.equal(a, b) for a, b in zip(begun, student.parameters()))
    assert len(losses) == 6 and all(torch.isfinite(torch.tensor(losses)))
    assert decoder.generate(student, decoder.repeating(2, 8, 50, torch.Generator(device="cuda").manual_seed(3))[:, :9], 5).shape == (2, 14)


def test_a_students_gradients(decoder):
    """distill's loss on the student's logits, against differences."""
    from paper_2601_15473_amd.block import distillation_loss
    teacher, student = decoder.Decoder(**SIZES, dtype=torch.float32, dense=True).eval(), decoder.Decoder(**SIZES, rank=64, dtype=torch.float32, seed=5, p=0.0).eval()
    ids = _ids(4, 12)
    with torch.no_grad():
        values, places = teacher(ids).topk(8, -1)
    loss = lambda: distillation_loss(student(ids), values, places, ids.roll(-1, 1), temperature=2.0, label_weight=0.3).double().sum()  # noqa: E731
    grads = torch.autograd.grad(loss(), list(student.parameters()))
    with torch.no_grad():
        for i, (w, g) in enumerate(zip(student.parameters(), grads)):
            v = g / g.norm().clamp(min=1e-6)         # the steepest way: the slope is the gradient's size
            h = 2.0 ** -7 * max(w.norm().item() / w.numel() ** 0.5, 2.0 ** -6)
            f = []
            for k in (1, -1):
                w.add_(k * h * v)
                f.append(loss().item())
                w.add_(-k * h * v)
            slope = (f[0] - f[1]) / (2 * h)
            # h^2 of a third derivative, and the roundings of 48 losses of order ten (some 200 terms' each) over 2 h
            assert abs(slope - g.norm().item()) <= 0.03 * g.norm().item() + 48 * 10 * 200 * 2.0 ** -24 / (2 * h), i
