"""Beam search on a head by itself where rows of the head are zeros, as of a padded
vocabulary."""
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams", [1, 4])
def test_zero_rows_of_the_head(sq, torch, beams):  # noqa: F811
    # logits of the other tokens are negative, so the padded ones are the likeliest
    from paper_2609_38477_amd import scoring
    W, h, _ = scoring.sample(600, 128, 5)
    W = torch.where((h[:1] @ W.t()).t() < 0, W, -W)
    W = torch.cat([W, torch.zeros(8, 128, device="cuda")])
    h = h[:1].repeat(5, 1)
    found, score = scoring.continuations(lambda x: x @ W.t(), W, h, beams, 6)
    assert (found[:, 0, 0] >= 600).all()
    assert (found >= 0).all() and (found < 608).all() and torch.isfinite(score).all()
    # a state that a row of zeros leaves as it is: the same logits at every step
    first = torch.log_softmax((h @ W.t()).double(), 1).max(1).values
    if beams == 1:
        assert (found >= 600).all() and torch.allclose(score[:, 0].double(), 6 * first, atol=1e-4)
