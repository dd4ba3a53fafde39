"""Results whose rows lie on one another are refused before any launch: threads would write the same place in no order."""
import itertools

import pytest

from paper_2601_15473_amd import libsk as sk

P = 0x100000000


def _call(tokens, heads, kv_heads, D, q_out, k_out):
    s = sk.NormRopeShape(tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=D, rotary_dim=8, position_bytes=8, table_rows=9, eps=1e-6, dtype=sk.SK_F32)
    s.q_strides[:], s.k_strides[:] = (0, 0), (0, 0)          # (inputs may be expanded)
    s.q_out_strides[:], s.k_out_strides[:] = q_out, k_out
    sk.sk_trace_begin()
    try:
        return sk.sk_norm_rope_fwd(s, *(P,) * 9)
    finally:
        sk.sk_trace_end()


@pytest.mark.parametrize("tokens, heads", [(1, 1), (1, 4), (3, 1), (2, 2), (3, 4), (5, 3)])
def test_rows_that_overlap(tokens, heads):
    """Against every pair of rows, over strides of 0 to 8 half heads each."""
    D = 8
    for a, b in itertools.product(range(0, 9 * 4, 4), repeat=2):
        begins = [t * a + h * b for t in range(tokens) for h in range(heads)]
        overlap = any(abs(x - y) < D for i, x in enumerate(begins) for y in begins[:i])
        want = sk.SK_ERR_INVALID_ARG if overlap else sk.SK_OK
        dense = (heads * D, D)
        assert _call(tokens, heads, heads, D, (a, b), dense) == want, (a, b)
        assert _call(tokens, heads, heads, D, dense, (a, b)) == want, (a, b)
        assert _call(tokens, heads, 0, D, dense, (a, b)) == sk.SK_OK


def test_slices_of_a_tensor():
    for q_out, k_out in (((72 * 64, 64), (72 * 64, 64)), ((64, 1000 * 64), (128, 2000 * 64)), ((1 << 20, 64), (128, 1 << 22))):
        assert _call(1000, 64, 8, 64, q_out, k_out) == sk.SK_OK
