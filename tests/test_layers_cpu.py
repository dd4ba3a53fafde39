"""Layer norm, dense layers and the distillation loss without a GPU: refusals before any HIP call, and every access of every launch inside the caller's
buffers, at the smallest and the largest sizes too."""
import ctypes
import math
import random

import pytest

from paper_2601_15473_amd import libsk as sk
from test_block_cpu import BIG, NONE, P, Buffers, traced


def norm_shape(rows=5, width=64, eps=1e-5, dtype=sk.SK_BF16, x_stride=None, residual_stride=None):
    return sk.LayerNormShape(rows, width, eps, dtype, width if x_stride is None else x_stride, width if residual_stride is None else residual_stride)


def dense_shape(tokens=5, d_in=64, d_out=48, activation=sk.SK_ACT_GELU, dtype=sk.SK_BF16, x_stride=None, residual_stride=None):
    return sk.DenseShape(tokens, d_in, d_out, activation, dtype, d_in if x_stride is None else x_stride, d_out if residual_stride is None else residual_stride)


def distill_shape(rows=5, vocabulary=77, logits_stride=None, top=6, id_bytes=4, label_bytes=8, temperature=1.0, label_weight=0.5, dtype=sk.SK_BF16):
    return sk.DistillShape(rows, vocabulary, vocabulary if logits_stride is None else logits_stride, top, id_bytes, label_bytes, temperature, label_weight, dtype)


def test_shapes_have_the_headers_layout():
    assert ctypes.sizeof(sk.LayerNormShape) == 2 * 8 + 4 + 4 + 2 * 8
    assert ctypes.sizeof(sk.DenseShape) == 3 * 8 + 4 + 4 + 2 * 8
    assert ctypes.sizeof(sk.DistillShape) == 3 * 8 + 3 * 4 + 2 * 4 + 4


@pytest.mark.parametrize("change, want", [
    (dict(rows=0), 1), (dict(width=0), 1), (dict(width=-8), 1), (dict(eps=-1.0), 1), (dict(eps=math.nan), 1), (dict(eps=math.inf), 1), (dict(x_stride=-64), 1), (dict(residual_stride=-64), 1),
    (dict(width=60), 2), (dict(width=(1 << 15) + 8), 2), (dict(rows=1 << 24), 2), (dict(rows=1 << 22, width=8200), 2), (dict(dtype=4), 2), (dict(x_stride=68), 2), (dict(x_stride=(1 << 40) + 8), 2), (dict(residual_stride=65), 2),
])
def test_layer_norm_refusals(change, want):
    s = norm_shape(**change)
    assert sk.sk_layer_norm_fwd(s, *(P,) * 7) == want
    assert sk.sk_layer_norm_bwd(s, *(P,) * 8, P, BIG) == want
    assert sk.sk_layer_norm_workspace_bytes(s) == NONE


def test_layer_norm_pointers_and_workspace():
    s = norm_shape()
    need = sk.sk_layer_norm_workspace_bytes(s)
    assert 0 < need < 1 << 20
    for i in range(7):
        args = [P] * 7
        args[i] = P + 8
        assert sk.sk_layer_norm_fwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i not in (0, 4) or sk.sk_layer_norm_fwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
    for i in range(8):
        args = [P] * 8
        args[i] = P + 8
        assert sk.sk_layer_norm_bwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i not in (0, 2, 3, 5) or sk.sk_layer_norm_bwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
    assert sk.sk_layer_norm_bwd(s, *(P,) * 8, P, need - 1) == sk.sk_layer_norm_bwd(s, *(P,) * 8, None, 0) == sk.SK_ERR_WORKSPACE
    assert sk.sk_layer_norm_fwd(None, *(P,) * 7) == sk.SK_ERR_INVALID_ARG
    # what a sum's rounding left off: of a sum, in bf16, from a boundary on
    assert sk.sk_layer_norm_fwd(s, *(P,) * 5, None, P, sum_rest=P) == sk.SK_ERR_INVALID_ARG
    assert sk.sk_layer_norm_fwd(s, *(P,) * 7, sum_rest=P + 4) == sk.sk_layer_norm_bwd(s, *(P,) * 8, P, BIG, sum_rest=P + 4) == sk.SK_ERR_INVALID_ARG
    f32 = norm_shape(dtype=sk.SK_F32)
    assert sk.sk_layer_norm_fwd(f32, *(P,) * 7, sum_rest=P) == sk.sk_layer_norm_bwd(f32, *(P,) * 8, P, BIG, sum_rest=P) == sk.SK_ERR_INVALID_ARG


@pytest.mark.parametrize("change, want", [
    (dict(tokens=0), 1), (dict(d_in=0), 1), (dict(d_out=-8), 1), (dict(activation=-1), 1), (dict(x_stride=-64), 1),
    (dict(activation=5), 2), (dict(d_in=60), 2), (dict(d_out=44), 2), (dict(tokens=(1 << 24) + 1), 2), (dict(d_in=(1 << 20) + 8), 2), (dict(d_out=(1 << 20) + 8), 2), (dict(dtype=9), 2),
    (dict(x_stride=56), 2), (dict(x_stride=0), 2), (dict(x_stride=68), 2), (dict(residual_stride=40), 2), (dict(x_stride=(1 << 20) + 8), 2), (dict(residual_stride=(1 << 20) + 8), 2),
    (dict(tokens=1 << 24, d_in=1024), 2), (dict(d_in=1 << 20, d_out=1 << 14), 2),
])
def test_dense_refusals(change, want):
    s = dense_shape(**change)
    assert sk.sk_dense_fwd(s, *(P,) * 6, P, BIG) == want
    assert sk.sk_dense_bwd(s, *(P,) * 7, P, BIG) == want
    assert sk.sk_dense_workspace_bytes(s, 0) == NONE and sk.sk_dense_workspace_bytes(s, 1) == NONE


def test_dense_pointers_and_workspace():
    s = dense_shape()
    for i in range(6):
        args = [P] * 6
        args[i] = P + 8
        assert sk.sk_dense_fwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i not in (0, 1, 4) or sk.sk_dense_fwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
    for i in range(7):
        args = [P] * 7
        args[i] = P + 8
        assert sk.sk_dense_bwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i not in (0, 1, 2, 3) or sk.sk_dense_bwd(s, *args, P, BIG) == sk.SK_ERR_INVALID_ARG, i
    assert sk.sk_dense_fwd(None, *(P,) * 6, P, BIG) == sk.SK_ERR_INVALID_ARG
    for shape in (dense_shape(tokens=8, d_in=8192, d_out=64), dense_shape(tokens=100, d_in=64, d_out=64, dtype=sk.SK_F32), s):
        need = sk.sk_dense_workspace_bytes(shape, 1)
        assert need > 0 and sk.sk_dense_bwd(shape, *(P,) * 7, P, need - 1) == sk.sk_dense_bwd(shape, *(P,) * 7, None, 0) == sk.SK_ERR_WORKSPACE
        need = sk.sk_dense_workspace_bytes(shape, 0)
        if need > 0:
            assert sk.sk_dense_fwd(shape, *(P,) * 6, P, need - 1) == sk.sk_dense_fwd(shape, *(P,) * 6, None, 0) == sk.SK_ERR_WORKSPACE


@pytest.mark.parametrize("change, want", [
    (dict(rows=0), 1), (dict(vocabulary=0), 1), (dict(top=-1), 1), (dict(logits_stride=-1), 1), (dict(temperature=0.0), 1), (dict(temperature=-1.0), 1), (dict(temperature=math.nan), 1),
    (dict(temperature=math.inf), 1), (dict(label_weight=-0.1), 1), (dict(label_weight=1.1), 1), (dict(label_weight=math.nan), 1),
    (dict(dtype=2), 2), (dict(id_bytes=2), 2), (dict(label_bytes=1), 2), (dict(rows=1 << 23), 2), (dict(vocabulary=(1 << 24) + 1), 2), (dict(top=(1 << 16) + 1), 2), (dict(temperature=1e-4), 2),
    (dict(temperature=2e3), 2), (dict(logits_stride=(1 << 40) + 1), 2),
])
def test_distill_refusals(change, want):
    s = distill_shape(**change)
    assert sk.sk_distill_fwd(s, *(P,) * 6) == want
    assert sk.sk_distill_bwd(s, *(P,) * 7) == want


def test_distill_pointers():
    s = distill_shape()
    for i in range(6):
        args = [P] * 6
        args[i] = P + (8 if i else 1)      # (rows of logits begin anywhere that a value does)
        assert sk.sk_distill_fwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i in (3, 5) or sk.sk_distill_fwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
    for i in range(7):
        args = [P] * 7
        args[i] = P + (8 if i else 1)
        assert sk.sk_distill_bwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
        args[i] = None
        assert i == 3 or sk.sk_distill_bwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
    assert sk.sk_distill_fwd(None, *(P,) * 6) == sk.SK_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype, e", [(sk.SK_BF16, 2), (sk.SK_F32, 4)], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows, width", [(1, 8), (3, 64), (1000, 72), (5000, 768), (16384, 4096), (7, 32768), ((1 << 24) - 1, 8), ((1 << 24) - 1, 8192), ((1 << 22) - 1, 32768)])
def test_layer_norm_accesses(rows, width, dtype, e):
    for residual in (False, True):
        buf = Buffers()
        s = norm_shape(rows, width, dtype=dtype, x_stride=width + 16)
        x, r = buf.new(((rows - 1) * (width + 16) + width) * e), buf.new(rows * width * e) if residual else None
        w, b, y, stats = buf.new(width * e), buf.new(width * e), buf.new(rows * width * e, both=True), buf.new(rows * 8, both=True)
        total = buf.new(rows * width * e, both=True) if residual else None
        buf.check(traced(lambda: sk.sk_layer_norm_fwd(s, x, r, w, b, y, total, stats))[0])
        rest = buf.new(rows * width // 2, both=True) if residual and dtype == sk.SK_BF16 else None
        buf.check(traced(lambda: sk.sk_layer_norm_fwd(s, x, r, w, b, y, total, stats, sum_rest=rest))[0])
        need = sk.sk_layer_norm_workspace_bytes(s)
        dy, ds = buf.new(rows * width * e), buf.new(rows * width * e) if residual else None
        out = buf.new(rows * width * e, write=True), buf.new(width * e, write=True), buf.new(width * e, write=True)
        ws = buf.new(need, both=True)
        accesses, launches = traced(lambda: sk.sk_layer_norm_bwd(s, x, w, stats, dy, ds, *out, ws, need, sum_rest=rest))
        buf.check(accesses)
        assert launches == (2 if width <= 8192 else 3) and traced(lambda: sk.sk_layer_norm_bwd(s, x, w, stats, dy, ds, out[0], None, None, None, 0))[1] == 1


def _dense_accesses(tokens, d_in, d_out, dtype, e, act, x_stride):
    buf = Buffers()
    s = dense_shape(tokens, d_in, d_out, act, dtype, x_stride)
    x, w, b, r = buf.new(((tokens - 1) * x_stride + d_in) * e), buf.new(d_out * d_in * e), buf.new(d_out * e), buf.new(tokens * d_out * e)
    y, z = buf.new(tokens * d_out * e, write=True), buf.new(tokens * d_out * e, both=True)
    need = sk.sk_dense_workspace_bytes(s, 0)
    ws = buf.new(need, both=True) if need else None
    for pre in (z, None):
        for residual in (r, None):
            buf.check(traced(lambda: sk.sk_dense_fwd(s, x, w, b, residual, y, pre, ws, need))[0])
    need = sk.sk_dense_workspace_bytes(s, 1)
    ws, dy = buf.new(need, both=True), buf.new(tokens * d_out * e)
    grads = [buf.new(n * e, write=True) for n in (tokens * d_in, d_out * d_in, d_out)]
    for which in range(1, 8):
        buf.check(traced(lambda: sk.sk_dense_bwd(s, x, w, z, dy, *(g if which >> i & 1 else None for i, g in enumerate(grads)), ws, need))[0])


@pytest.mark.parametrize("dtype, e", [(sk.SK_BF16, 2), (sk.SK_F32, 4)], ids=["bf16", "f32"])
def test_dense_accesses(dtype, e):
    rng = random.Random(2)
    sizes = [(1, 8, 8), (8, 4096, 11008), (8, 11008, 4096), (4001, 4096, 1024), (4096, 1024, 4096), (16384, 4096, 11008), (1 << 24, 8, 8), (1, 1 << 20, 8), (1, 8, 1 << 20), (64, 256, 256)]
    sizes += [(max(1, int(2 ** rng.uniform(0, 15))), 8 * max(1, int(2 ** rng.uniform(0, 10))), 8 * max(1, int(2 ** rng.uniform(0, 10)))) for _ in range(150)]
    for tokens, d_in, d_out in sizes:
        for act in (sk.SK_ACT_NONE, sk.SK_ACT_SILU):
            stride = rng.choice([d_in, d_in, d_in + 8, d_in + 264, 1 << 20])
            _dense_accesses(tokens, d_in, d_out, dtype, e, act, stride if stride <= 1 << 20 else d_in)


@pytest.mark.parametrize("dtype", [sk.SK_F32, sk.SK_BF16])
def test_dense_layers_of_the_most_values(dtype):
    """Every launch of the largest calls is one that HIP takes (the trace refuses the others)."""
    most = (1 << 34) - 1
    for tokens, d_in, d_out in ((1 << 24, 1016, 1016), (1 << 24, 8, 1016), (1 << 24, 1016, 8), (16376, 1 << 20, 8), (16376, 8, 1 << 20), (8, 16376, 1 << 20), (8, 1 << 20, 16376), (1 << 17, 131064, 8)):
        assert max(tokens * d_in, tokens * d_out, d_in * d_out) <= most
        for act in (0, 2):
            s = dense_shape(tokens, d_in, d_out, act, dtype)
            assert traced(lambda: sk.sk_dense_fwd(s, *(1 << 44,) * 6, 1 << 44, 1 << 62))[1] > 0, (tokens, d_in, d_out)
            assert traced(lambda: sk.sk_dense_bwd(s, *(1 << 44,) * 7, 1 << 44, 1 << 62))[1] > 0, (tokens, d_in, d_out)


@pytest.mark.parametrize("dtype, e", [(sk.SK_BF16, 2), (sk.SK_F32, 4)], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows, vocabulary, top", [(1, 1, 1), (3, 7, 0), (1000, 64, 8), (4001, 32001, 64), (5, 1 << 24, 1 << 16), ((1 << 23) - 1, 50, 3), ((1 << 23) - 1, 50000, 3)])
def test_distill_accesses(rows, vocabulary, top, dtype, e):
    for labels in (False, True):
        buf = Buffers()
        s = distill_shape(rows, vocabulary, vocabulary + 3, top, temperature=2.0, dtype=dtype)
        z = buf.new(((rows - 1) * (vocabulary + 3) + vocabulary) * e)
        t, ids = (buf.new(rows * top * e), buf.new(rows * top * 4)) if top else (None, None)
        y = buf.new(rows * 8) if labels else None
        loss, stats = buf.new(rows * 4, write=True), buf.new(rows * 32, both=True)
        buf.check(traced(lambda: sk.sk_distill_fwd(s, z, t, ids, y, loss, stats))[0])
        dz = buf.new(rows * vocabulary * e, write=True)
        buf.check(traced(lambda: sk.sk_distill_bwd(s, z, t, ids, y, stats, buf.new(rows * 4), dz))[0])
