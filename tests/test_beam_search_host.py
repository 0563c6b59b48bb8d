"""Beam search where nothing is searched, on the host."""
import pytest


@pytest.mark.parametrize("batch,beams", [(3, 1), (2, 4), (1, 32)])
def test_no_tokens_at_all(batch, beams):
    import torch
    from paper_2609_38477_amd import scoring

    def step(tokens, states):
        raise AssertionError("there is no step")

    found, score = scoring.beam_search(step, [], torch.zeros(batch, dtype=torch.int64), beams, 0)
    assert found.shape == (batch, beams, 0) and score.shape == (batch, beams)
    assert (score[:, 0] == 0).all() and (score[:, 1:] == float("-inf")).all()
