"""More tokens than one dimension of a launch has work-groups for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_rows_past_one_dimension_of_work_groups():
    from paper_2601_15473_amd import block
    width, tokens = 520, (1 << 25) + 4 * 100 + 3        # (four rows to a work-group: 2^23 of them and a hundred)
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("70 GB of results do not fit")
    g = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn(100, width, generator=g, device="cuda")
    ids = torch.randint(-3, 103, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    y = block.embedding(ids, table, 2.0)
    for at in (0, (1 << 25) - 200, tokens - 300):
        i = ids[at:at + 300].long()
        want = torch.where(((i >= 0) & (i < 100))[:, None], 2 * table[i.clamp(0, 99)], 0.0)
        assert torch.equal(y[at:at + 300], want[:len(y) - at])
