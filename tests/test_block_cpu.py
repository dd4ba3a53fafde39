"""The block operators' C ABI without a GPU: exports, refusals before any HIP call, and every access inside the caller's buffers."""
import ctypes
import math
import os
import re

import pytest

from paper_2601_15473_amd import libsk as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x100000000
BIG = 1 << 40
NONE = 2 ** 64 - 1


def attention_shape(batch=2, q_len=10, k_len=12, heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, dtype=sk.SK_BF16, **more):
    s = sk.AttentionShape(batch=batch, q_len=q_len, k_len=k_len, heads=heads, kv_heads=kv_heads, head_dim=head_dim, causal=causal, scale=scale, dtype=dtype)
    s.q_strides[:] = (q_len * heads * head_dim, heads * head_dim, head_dim)
    s.k_strides[:] = s.v_strides[:] = (k_len * kv_heads * head_dim, kv_heads * head_dim, head_dim)
    for n, v in more.items():
        if isinstance(v, tuple):
            getattr(s, n)[:] = v
        else:
            setattr(s, n, v)
    return s


def norm_shape(tokens=5, heads=4, kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, position_bytes=8, table_rows=9, eps=1e-6, dtype=sk.SK_BF16, **more):
    s = sk.NormRopeShape(tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotary_dim=rotary_dim, interleaved=interleaved,
                         position_bytes=position_bytes, table_rows=table_rows, eps=eps, dtype=dtype)
    s.q_strides[:] = s.q_out_strides[:] = (heads * head_dim, head_dim)
    s.k_strides[:] = s.k_out_strides[:] = (kv_heads * head_dim, head_dim)
    for n, v in more.items():
        getattr(s, n)[:] = v
    return s


def fwd(s, q=P, k=P, v=P, o=P, lse=P, rest=P, ws=P, n=BIG):
    return sk.sk_attention_fwd(s, q, k, v, o, lse, rest, ws, n)


def bwd(s, *ptrs, ws=P, n=BIG):
    ptrs = ptrs or (P,) * 9
    return sk.sk_attention_bwd(s, *ptrs[:5], P, *ptrs[5:], ws, n)


def test_every_declared_symbol_is_exported():
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sk_block.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(sk_[a-z_]+)\s*\(", hdr))
    assert declared == set(sk.BLOCK_EXPORTS)
    for name in declared:
        assert hasattr(sk._lib, name), name


@pytest.mark.parametrize("change, want", [
    (dict(batch=0), 1), (dict(q_len=0), 1), (dict(k_len=-1), 1), (dict(kv_heads=0), 1), (dict(head_dim=0), 1), (dict(scale=math.inf), 1), (dict(scale=math.nan), 1),
    (dict(causal=2), 1), (dict(q_strides=(-640, 256, 64)), 1), (dict(k_lengths=P + 2), 1),
    (dict(dtype=7), 2), (dict(head_dim=60), 2), (dict(head_dim=136), 2), (dict(heads=5), 2), (dict(q_strides=(2560, 256, 60)), 2),
    (dict(k_strides=(1 << 30, 1 << 23, 64)), 2), (dict(heads=1 << 17, kv_heads=1 << 17), 2), (dict(v_strides=(1 << 41, 128, 64)), 2), (dict(q_len=1 << 27), 2), (dict(k_len=(1 << 27) + 1), 2),
    (dict(batch=1 << 22, k_strides=(0, 0, 0), v_strides=(0, 0, 0), q_strides=(0, 0, 0)), 2),
])
def test_attention_refusals(change, want):
    s = attention_shape(**change)
    assert fwd(s) == want and bwd(s) == want
    if want == 2 or "k_lengths" not in change:
        assert sk.sk_attention_workspace_bytes(s, 0) == NONE and sk.sk_attention_workspace_bytes(s, 1) == NONE


def test_attention_pointers_and_workspace():
    s = attention_shape()
    for i in range(4):
        for bad in (None, P + 8):
            args = [P] * 4
            args[i] = bad
            assert fwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
    assert fwd(s, lse=P + 4) == fwd(s, rest=P + 8) == sk.SK_ERR_INVALID_ARG and sk.sk_attention_fwd(None, P, P, P, P, P, P, P, BIG) == sk.SK_ERR_INVALID_ARG
    for i in range(9):
        args = [P] * 9
        args[i] = None
        assert bwd(s, *args) == sk.SK_ERR_INVALID_ARG, i
    need = sk.sk_attention_workspace_bytes(s, 1)
    assert need >= 2 * 4 * 10 * 4
    assert bwd(s, n=need - 1) == sk.SK_ERR_WORKSPACE and bwd(s, ws=None) == sk.SK_ERR_WORKSPACE


@pytest.mark.parametrize("change, want", [
    (dict(tokens=0), 1), (dict(heads=0), 1), (dict(kv_heads=-1), 1), (dict(rotary_dim=72), 1), (dict(eps=-1.0), 1), (dict(eps=math.nan), 1), (dict(table_rows=0), 1),
    (dict(interleaved=2), 1), (dict(q_strides=(-64, 64)), 1),
    (dict(dtype=3), 2), (dict(head_dim=68, rotary_dim=0), 2), (dict(head_dim=264), 2), (dict(rotary_dim=12), 2), (dict(position_bytes=2), 2), (dict(q_strides=(260, 60)), 2),
])
def test_norm_rope_refusals(change, want):
    s = norm_shape(**change)
    assert sk.sk_norm_rope_fwd(s, *(P,) * 9) == want
    assert sk.sk_norm_rope_bwd(s, *(P,) * 13, P, BIG) == want
    assert sk.sk_norm_rope_workspace_bytes(s) == NONE
    assert sk.sk_norm_rope_fwd(norm_shape(), *(P,) * 8, None) == sk.SK_ERR_INVALID_ARG
    assert sk.sk_norm_rope_bwd(norm_shape(), *(P,) * 13, P, 16) == sk.SK_ERR_WORKSPACE


@pytest.mark.parametrize("tokens, rows, width, scale, dtype, id_bytes, want", [
    (0, 5, 16, 1.0, 1, 8, 1), (3, 0, 16, 1.0, 1, 8, 1), (3, 5, 0, 1.0, 1, 8, 1), (3, 5, 16, math.inf, 1, 8, 1),
    (3, 5, 12, 1.0, 1, 8, 2), (3, 1 << 31, 16, 1.0, 1, 8, 2), (1 << 28, 5, 16, 1.0, 1, 8, 2), (3, 5, 16, 1.0, 9, 8, 2), (3, 5, 16, 1.0, 1, 2, 2),
])
def test_embedding_refusals(tokens, rows, width, scale, dtype, id_bytes, want):
    assert sk.sk_embedding_fwd(P, id_bytes, P, P, tokens, rows, width, scale, dtype) == want
    assert sk.sk_embedding_bwd(P, id_bytes, P, P, tokens, rows, width, scale, dtype, P, BIG) == want
    if scale == 1.0 and id_bytes == 8:
        assert sk.sk_embedding_workspace_bytes(tokens, rows, width, dtype) == NONE
    need = sk.sk_embedding_workspace_bytes(100, 5, 16, 1)
    assert sk.sk_embedding_bwd(P, 8, P, P, 100, 5, 16, 1.0, 1, P, need - 1) == sk.SK_ERR_WORKSPACE
    assert sk.sk_embedding_fwd(P + 8, 8, P, P, 100, 5, 16, 1.0, 1) == sk.SK_ERR_INVALID_ARG


def test_dropout_refusals():
    for p in (-0.1, 1.1, math.nan):
        assert sk.sk_dropout(P, None, P, 4, p, 1, 0, sk.SK_F32) == sk.SK_ERR_INVALID_ARG
    assert sk.sk_dropout(P, None, P, 0, 0.5, 1, 0, sk.SK_F32) == sk.SK_ERR_INVALID_ARG
    assert sk.sk_dropout(P, P + 4, P, 4, 0.5, 1, 0, sk.SK_F32) == sk.SK_ERR_INVALID_ARG
    assert sk.sk_dropout(P, None, P, 4, 0.5, 1, 0, 5) == sk.SK_ERR_UNSUPPORTED


# ---- where the launches read and write ----

class Buffers:
    """Made-up buffers far apart; every recorded access has to lie in one, in the direction it may."""

    def __init__(self):
        self.at, self.held = 1 << 40, []

    def new(self, nbytes, write=False, both=False):
        p = self.at
        self.held.append((p, p + nbytes, write or both, not write or both))
        self.at += (nbytes + (1 << 30)) // 256 * 256
        return p

    def check(self, accesses):
        assert accesses
        for address, nbytes, write, launch in accesses:
            assert any(a <= address and address + nbytes <= b and (w if write else r) for a, b, w, r in self.held), (address, nbytes, write, launch)


def traced(call):
    sk.sk_trace_begin()
    try:
        status = call()
    finally:
        accesses, launches = sk.sk_trace_end()
    assert status == sk.SK_OK
    return accesses, launches


ATTENTION = [(1, 1, 1, 1, 1, 8), (2, 1, 5000, 64, 8, 128), (32, 128, 128, 12, 12, 64), (4, 4096, 4096, 32, 8, 128), (1, 1001, 3001, 64, 8, 128), (3, 17, 100, 6, 2, 80),
             (1, 2, 32768, 8, 1, 96), (7, 1, 33, 5, 5, 32),
             (1, 4096, 4096, 4, 2, 64), (2, 2292, 2292, 4, 1, 32), (4, 300, 4000, 8, 2, 128), (1, 2493, 2493, 1, 1, 64), (3, 3875, 3875, 4, 1, 128), (1, 55, 55, 4, 1, 40)]


@pytest.mark.parametrize("dtype, e", [(sk.SK_BF16, 2), (sk.SK_F32, 4)], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", ATTENTION, ids=lambda s: "x".join(map(str, s)))
def test_attention_accesses(shape, dtype, e):
    B, Tq, Tk, H, Hkv, D = shape
    buf = Buffers()
    s = attention_shape(*shape, dtype=dtype, q_lengths=buf.new(4 * B), k_lengths=buf.new(4 * B))
    rows, keys = B * Tq * H, B * Tk * Hkv * D * e
    q, k, v = buf.new(rows * D * e), buf.new(keys), buf.new(keys)
    o, lse, rest = buf.new(rows * D * e, both=True), buf.new(rows * 4, both=True), buf.new(rows * D * e, both=True)
    need = sk.sk_attention_workspace_bytes(s, 0)
    accesses, launches = traced(lambda: sk.sk_attention_fwd(s, q, k, v, o, lse, rest, buf.new(need, both=True), need))
    buf.check(accesses)
    assert 1 <= launches <= 2
    need = sk.sk_attention_workspace_bytes(s, 1)
    grads = buf.new(rows * D * e), buf.new(rows * D * e, write=True), buf.new(keys, write=True), buf.new(keys, write=True)
    accesses, launches = traced(lambda: sk.sk_attention_bwd(s, q, k, v, o, lse, rest, *grads, buf.new(need, both=True), need))
    buf.check(accesses)


@pytest.mark.parametrize("tokens, rows, width", [(1, 1, 8), (33, 5, 16), (16384, 65536, 4096), (16385, 100, 8), (1 << 20, 1 << 17, 64)])
def test_embedding_accesses(tokens, rows, width):
    buf = Buffers()
    ids, dy, dt = buf.new(8 * tokens), buf.new(2 * tokens * width), buf.new(2 * rows * width, write=True)
    need = sk.sk_embedding_workspace_bytes(tokens, rows, width, sk.SK_BF16)
    ws = buf.new(need, both=True)
    accesses, launches = traced(lambda: sk.sk_embedding_bwd(ids, 8, dy, dt, tokens, rows, width, 1.0, sk.SK_BF16, ws, need))
    buf.check(accesses)
    assert launches <= 4


@pytest.mark.parametrize("kv_heads", [0, 2])
@pytest.mark.parametrize("tokens", [1, 5, 16384])
def test_norm_rope_accesses(tokens, kv_heads):
    buf = Buffers()
    s = norm_shape(tokens=tokens, kv_heads=kv_heads)
    q, k = buf.new(tokens * 4 * 64 * 2), buf.new(tokens * kv_heads * 64 * 2)
    w = [buf.new(128) for _ in range(2)]
    tables = [buf.new(9 * 32 * 4) for _ in range(2)] + [buf.new(8 * tokens)]
    out = buf.new(tokens * 4 * 64 * 2, write=True), buf.new(tokens * kv_heads * 64 * 2, write=True)
    buf.check(traced(lambda: sk.sk_norm_rope_fwd(s, q, k, *w, *tables, *out))[0])
    need = sk.sk_norm_rope_workspace_bytes(s)
    grads = buf.new(tokens * 4 * 64 * 2), buf.new(tokens * kv_heads * 64 * 2), *out, buf.new(128, write=True), buf.new(128, write=True)
    buf.check(traced(lambda: sk.sk_norm_rope_bwd(s, q, k, *w, *tables, *grads, buf.new(need, both=True), need))[0])


def test_shapes_have_the_headers_layout():
    """The structures' sizes on this ABI, as include/sk_block.h lays them out."""
    assert ctypes.sizeof(sk.AttentionShape) == 3 * 8 + 4 * 4 + 4 + 4 + 9 * 8 + 2 * 8
    assert ctypes.sizeof(sk.NormRopeShape) == 8 + 6 * 4 + 8 + 4 + 4 + 8 * 8
