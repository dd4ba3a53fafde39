"""The largest calls that include/sk_block.h takes: every launch of theirs is one that HIP takes too, and stays inside the buffers."""
import random

import pytest

from paper_2601_15473_amd import libsk as sk

P = 1 << 44
BIG = 1 << 62


def _traced(call):
    sk.sk_trace_begin()
    try:
        status = call()
        kernels = sk.sk_trace_kernels()
    finally:
        sk.sk_trace_end()
    return status, kernels


def _embeddings():
    """Token counts up to the last that a width takes, by its workspace's size."""
    rng = random.Random(0)
    widths = [8, 64, 128, 256, 264, 512, 520, 768, 776, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 1 << 20] + [8 * rng.randrange(1, 2000) for _ in range(20)]
    for width in widths:
        for dtype in (sk.SK_F32, sk.SK_BF16):
            lo, hi = 1, 1 << 27
            while lo < hi:
                mid = (lo + hi + 1) // 2
                if sk.sk_embedding_workspace_bytes(mid, 100, width, dtype) != 2 ** 64 - 1:
                    lo = mid
                else:
                    hi = mid - 1
            yield width, dtype, lo


@pytest.mark.parametrize("width, dtype, most", list(_embeddings()))
def test_embeddings_of_the_most_tokens(width, dtype, most):
    for tokens in (most, most * 2 // 3 + 1, most // 2):
        assert _traced(lambda: sk.sk_embedding_fwd(P, 8, P, P, tokens, 100, width, 1.0, dtype))[0] == sk.SK_OK, tokens
        assert _traced(lambda: sk.sk_embedding_bwd(P, 8, P, P, tokens, 100, width, 1.0, dtype, P, BIG))[0] == sk.SK_OK, tokens


@pytest.mark.parametrize("dtype", [sk.SK_F32, sk.SK_BF16])
def test_attention_of_the_most_work_groups(dtype):
    rng = random.Random(1)
    taken = 0
    for _ in range(400):
        kv, group, D = rng.choice([1, 2, 8, 40]), rng.choice([1, 4, 16]), rng.choice([8, 64, 128])
        q, k, b = (int(2 ** rng.uniform(0, 27)), int(2 ** rng.uniform(0, 27)), int(2 ** rng.uniform(0, 23)))
        s = sk.AttentionShape(batch=b, q_len=q, k_len=k, heads=kv * group, kv_heads=kv, head_dim=D, causal=rng.randrange(2), scale=1.0, dtype=dtype)
        s.q_strides[:], s.k_strides[:], s.v_strides[:] = ((0, kv * group * D, D), (0, kv * D, D), (0, kv * D, D))
        if sk.sk_attention_workspace_bytes(s, 1) == 2 ** 64 - 1:
            continue
        taken += 1
        assert _traced(lambda: sk.sk_attention_fwd(s, P, P, P, P, P, P, P, BIG))[0] == sk.SK_OK, (b, q, k, kv, group, D)
        assert _traced(lambda: sk.sk_attention_bwd(s, *(P,) * 10, P, BIG))[0] == sk.SK_OK, (b, q, k, kv, group, D)
    assert taken > 50


def test_norms_and_dropout_of_the_most_tokens():
    for heads, kv, D in ((1, 0, 8), (1 << 16, 1 << 16, 256), (32, 8, 128)):
        s = sk.NormRopeShape(tokens=1 << 25, heads=heads, kv_heads=kv, head_dim=D, rotary_dim=8, position_bytes=8, table_rows=9, eps=1e-6, dtype=sk.SK_BF16)
        s.q_strides[:], s.q_out_strides[:] = (heads * D, D), (heads * D, D)
        s.k_strides[:], s.k_out_strides[:] = (kv * D, D), (kv * D, D)
        assert _traced(lambda: sk.sk_norm_rope_fwd(s, *(P,) * 9))[0] == sk.SK_OK
        assert _traced(lambda: sk.sk_norm_rope_bwd(s, *(P,) * 13, P, BIG))[0] == sk.SK_OK
    assert _traced(lambda: sk.sk_dropout(P, P, P, 1 << 40, 0.5, 1, 0, sk.SK_F32))[0] == sk.SK_OK
