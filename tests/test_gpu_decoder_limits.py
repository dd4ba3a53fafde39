"""The example model says so where its cache or its positions end, before anything is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _model(context):
    from paper_2601_15473_amd import decoder
    return decoder.Decoder(rows=50, width=128, layers=1, heads=2, kv_heads=1, head_dim=32, hidden=128, rank=64, context=context, dtype=torch.float32).eval()


def _ids(n):
    return torch.randint(0, 50, (2, n), generator=torch.Generator().manual_seed(n)).cuda()


def test_a_full_cache():
    model = _model(64)
    cache = model.cache(2, 12)
    model.append(_ids(9), cache)
    held = [t.clone() for t in cache]
    with pytest.raises(ValueError, match="room for 12"):
        model.append(_ids(4), cache)
    assert all(torch.equal(a, b) for a, b in zip(cache, held))
    model.append(_ids(3), cache)
    assert cache[1].tolist() == [12, 12]
    with pytest.raises(ValueError):
        model.append(_ids(1), cache)
    cache[1].zero_()                             # emptied: the room is there again
    assert torch.equal(model.append(_ids(9), cache), model.append(_ids(9), model.cache(2, 9)))


def test_part_of_a_cache():
    """One sequence's part of it, as a plain pair."""
    model = _model(64)
    cache = model.cache(2, 12)
    part = cache[0][:, :1], cache[1][:1]
    want = model.append(_ids(9)[:1], model.cache(1, 12))
    assert torch.equal(model.append(_ids(9)[:1], part), want) and cache[1].tolist() == [9, 0]
    with pytest.raises(ValueError, match="4 tokens behind 9"):
        model.append(_ids(4)[:1], part)


def test_positions_end():
    from paper_2601_15473_amd import decoder
    model = _model(16)
    model(_ids(16))
    with pytest.raises(ValueError, match="positions for 16"):
        model(_ids(17))
    cache = model.cache(2, 40)
    model.append(_ids(16), cache)
    with pytest.raises(ValueError, match="positions for 16"):
        model.append(_ids(1), cache)
    with pytest.raises(ValueError):
        decoder.generate(model, _ids(10), 8)
    assert decoder.generate(model, _ids(10), 6).shape == (2, 16)
