"""The example model, trained as its command does, continues sequences as they began."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_it_continues_what_it_was_trained_on():
    from paper_2601_15473_amd import decoder
    model = decoder.Decoder(rows=64)
    decoder.train(model, 200)
    ids = decoder.repeating(8, 16, 64, torch.Generator(device="cuda").manual_seed(2))
    got = decoder.generate(model, ids[:, :17], 15)
    assert torch.equal(got[:, :17], ids[:, :17])
    assert (got[:, 17:] == ids[:, 17:]).float().mean().item() > 0.9
