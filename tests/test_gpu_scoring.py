"""Scoring where some rows have no token: the figures are those of the other rows.

Bars: means of the same fp32 terms in another order, 1e-12 in fp64; rho sums squares in
fp32, 1e-6 of each."""
import math

import numpy as np
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sample(sq):
    from paper_2609_38477_amd import scoring
    return scoring.sample(600, 128, 40)


def test_rows_without_a_token_do_not_count(sq, torch, sample):
    from paper_2609_38477_amd import scoring
    W, h, tokens = sample
    logits = h @ W.t()
    some = tokens.clone()
    some[::3] = -1
    some[1] = -100
    keep = some >= 0
    a = scoring.score(logits, some)
    b = scoring.score(logits[keep].contiguous(), some[keep].contiguous())
    for k in ("nll", "perplexity", "entropy"):
        assert abs(a[k] - b[k]) <= 1e-12 * abs(b[k]), k
    assert a["top"].shape == (40, 5) and torch.equal(a["top"][keep], b["top"])
    rho = scoring.measured_rho(W, logits, some)
    ref = scoring.measured_rho(W, logits[keep].contiguous(), some[keep].contiguous())
    assert np.allclose(rho, ref, rtol=1e-6, atol=0)
    # all rows asked: as before
    z = torch.log_softmax(logits.double(), 1).gather(1, tokens[:, None]).squeeze(1)
    assert abs(scoring.score(logits, tokens)["nll"] + z.mean().item()) < 1e-5


def test_no_token_and_no_distribution(sq, torch, sample):
    from paper_2609_38477_amd import scoring
    W, h, tokens = sample
    logits = h @ W.t()
    none = scoring.score(logits, torch.full_like(tokens, -1))
    assert all(math.isnan(none[k]) for k in ("nll", "perplexity", "entropy"))
    assert np.isnan(scoring.measured_rho(W, logits, torch.full_like(tokens, -1))).all()
    outside = tokens.clone()
    outside[3] = 600
    assert math.isnan(scoring.score(logits, outside)["perplexity"])
    barred = logits.clone()
    barred[2, tokens[2]] = float("-inf")
    assert scoring.score(barred, tokens)["perplexity"] == math.inf


def test_faults_in_the_row_of_the_first_token(sq, torch, sample):
    from paper_2609_38477_amd import scoring
    W, h, tokens = sample
    q = sq.q4_quantize(W, 64, zeros=True)
    late = tokens.clone()
    late[:2] = -1
    late[2] = 600
    rows = scoring.fault_study(q, h, late)
    row = int(tokens[3])
    clean = sq.q4_dequantize(q)
    for part, index, bit in (("codes", row * q.codes.shape[1], 0), ("scale", row * q.scale.shape[1], 0)):
        bad = sq.q4_dequantize(scoring.flip_bit(q, part, index, bit))
        n, p, eta = sq.footprint(clean, bad)
        assert any(r["N_flip"] == n and r["eta"] == eta for r in rows)
        assert (bad != clean).any(1).nonzero().flatten().tolist() == [row]
    with pytest.raises(ValueError):
        scoring.fault_study(q, h, torch.full_like(tokens, -1))
