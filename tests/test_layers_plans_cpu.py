"""Which kernels the dense layers' products run on (host trace, no GPU)."""
import math
import random

import pytest

import test_gpu_linear_variants as variants
from paper_2601_15473_amd import libsk as sk

BASE = 1 << 44      # made-up device addresses, far apart; never dereferenced


def kernels(tokens, d_in, d_out, which, activation=sk.SK_ACT_NONE, dtype=sk.SK_BF16, residual=False, z=False):
    """Names and work-groups of a layer's launches: "fwd", "dx" or "dw"."""
    P = [i * BASE for i in range(1, 9)]
    s = sk.DenseShape(tokens, d_in, d_out, activation, dtype, d_in, d_out)
    n = sk.sk_dense_workspace_bytes(s, 0 if which == "fwd" else 1)
    sk.sk_trace_begin()
    try:
        if which == "fwd":
            sk.check(sk.sk_dense_fwd(s, *P[:3], P[3] if residual else None, P[4], P[5] if z else None, P[6], n))
        else:
            sk.check(sk.sk_dense_bwd(s, P[0], P[1], P[2], P[3], P[4] if which == "dx" else None, P[5] if which == "dw" else None, None, P[7], n))
        return sk.sk_trace_kernels()
    finally:
        sk.sk_trace_end()


@pytest.mark.parametrize("tokens, d_in, d_out, want", [
    (1, 64, 64, "<1, 1, false>"), (8, 1024, 1024, "<1, 1, false>"), (8, 8192, 1024, "<1, 1, false>"), (16, 768, 768, "<2, 1, false>"), (32, 768, 1536, "<4, 1, false>"),
    (64, 512, 1024, "<8, 1, false>"), (64, 768, 2048, "<8, 1, false>"), (100, 768, 768, "<8, 1, false>"), (128, 384, 768, "<8, 1, false>"), (200, 1024, 512, "<8, 1, false>"),
    (256, 512, 512, "<8, 1, false>"),
])
def test_input_gradients_of_few_tokens(tokens, d_in, d_out, want):
    got = kernels(tokens, d_in, d_out, "dx")
    assert [n for n, _ in got] == ["gemm_bf16_few_rows_kernel" + want], got


@pytest.mark.parametrize("tokens, d_in, d_out", [(257, 512, 512), (256, 2048, 2048), (512, 1024, 4096), (8, 8224, 1024), (17, 32768, 1024), (64, 11008, 2048), (200, 2080, 512)])
def test_input_gradients_of_more_tokens(tokens, d_in, d_out):
    """... on the tiles, and so are those whose columns make more than a round of 32-column work-groups."""
    assert all("few_rows" not in n for n, _ in kernels(tokens, d_in, d_out, "dx"))


def test_input_gradients_over_many_features_in_ranges():
    assert [n.split("<")[0] for n, _ in kernels(8, 1024, 4096, "dx")] == ["gemm_bf16_few_rows_kernel", "reduce_to_bf16_kernel"]


@pytest.mark.parametrize("tokens, d_in, d_out", [(6144, 1536, 1536), (8192, 1408, 1536), (65536, 1536, 1536), (65536, 2048, 1280), (1 << 20, 1536, 1536), (49152, 2048, 1536), (6144, 1024, 1024),
                                                 (3000, 512, 1024)])
def test_weight_gradients_of_many_tokens_in_ranges(tokens, d_in, d_out):
    """... so that they have the chip, and no sum is one chain over all of them."""
    got = kernels(tokens, d_in, d_out, "dw")
    assert len(got) == 2 and got[1][0] == "reduce_to_bf16_kernel" and got[0][1] > 160, got


@pytest.mark.parametrize("tokens, d_in, d_out", [(1400, 256, 256), (2500, 512, 1024), (4096, 1024, 1024), (2048, 768, 768), (4096, 1536, 1536)])
def test_weight_gradients_of_few_tokens_in_one_range(tokens, d_in, d_out):
    assert [n.split("<")[0] for n, _ in kernels(tokens, d_in, d_out, "dw")] == ["gemm_bf16_kernel"]


def _variants(sizes, dtype):
    """The kernels of these layers' forward and backward products; apart those whose work-groups walk on to another tile, which have more to wait for."""
    seen = set()
    for T, I, O in sizes:
        for which, tiles in (("fwd", (T, O)), ("dx", (T, I)), ("dw", (O, I))):
            for name, _ in kernels(T, I, O, which, sk.SK_ACT_RELU if which == "fwd" else sk.SK_ACT_NONE, dtype, residual=True, z=True):
                walks = "256, 256" in name or "crew" in name or "far" in name
                seen.add((name, walks and -(-tiles[0] // 256) * -(-tiles[1] // 256) > 256))
    return seen


@pytest.mark.parametrize("dtype", [sk.SK_BF16, sk.SK_F32], ids=["bf16", "f32"])
def test_every_kernel_that_is_taken_has_a_tested_size(dtype):
    rng = random.Random(1)

    def size(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    drawn = [(size(1, 1 << 16), 8 * size(1, 2048), 8 * size(1, 2048)) for _ in range(4000)]
    tested = _variants(variants.SIZES if dtype == sk.SK_BF16 else variants.SIZES_F32, dtype)
    assert _variants(drawn, dtype) <= tested


def test_operands_past_two_gigabytes_have_a_tested_size():
    names = [kernels(*s, "dw")[0][0] for s in variants.SIZES_FAR]
    assert names == ["gemm_bf16_far_kernel<false, false, bf16>"] * 2 + ["gemm_bf16_far_kernel<false, false, float>"], names
