"""Totals of rows in which many logits lie as far below the largest as each other, so that all of
their terms err alike, against the oracle.

Bar: the exponential instruction errs by 8.49e-8 of its result at the most (over every fp32
argument of +-126), the sum of two terms by 2^-24 (5.97e-8), what is left out of a bfloat16
argument's rest by (48 x 4.9e-6)^2 / 2 (2.76e-8), and all else is in fp64: 1.75e-7 of the sum of
exponentials, which is what the total errs by, and 2^-24 of it where it becomes fp32."""
import numpy as np
import pytest

from oracle import beam as obeam
from test_gpu_q4 import TYPES, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu

BAR = 1.75e-7


def check(sq, torch, x, scores=None):  # noqa: F811
    beams = x.shape[0]
    scores = torch.zeros(1, beams) if scores is None else scores
    got = sq.beam_select(x.cuda(), scores.cuda(), 1)
    for i in range(beams):      # one sequence a row too, so that every row's sum shows
        row = sq.beam_select(x[i:i + 1].cuda(), scores[:, i:i + 1].contiguous().cuda(), 2)
        want = obeam.select(x[i:i + 1].double().numpy(), scores[0, i:i + 1].numpy(), None, 0, 2)
        for r in range(2):
            if np.isinf(want[r][0]):
                assert row.score[0, r].item() == want[r][0] and row.token[0, r] == -1
                continue
            assert abs(row.score[0, r].item() - want[r][0]) <= BAR + 2.0 ** -24 * 1.0001 * abs(want[r][0]), (i, r)
            assert row.token[0, r] == want[r][2]
    best = obeam.select(x.double().numpy(), scores[0].numpy(), None, 0, 2)
    assert abs(got.score.item() - best[0][0]) <= BAR + 2.0 ** -24 * 1.0001 * abs(best[0][0])
    if best[0][0] - best[1][0] > 4e-7:
        assert (got.parent.item(), got.token.item()) == best[0][1:]


@pytest.mark.parametrize("vocab,far", [(32000, 7.15), (131072, 11.15), (262144, 11.15), (3000, 5.7), (32003, 9.3)])
def test_one_logit_and_many_alike(sq, torch, vocab, far):  # noqa: F811
    top = torch.tensor([0.0, 5.3, -2.7, 1e-3, 17.9, -60.1, 900.7])
    x = (top - far)[:, None].repeat(1, vocab)
    x[:, vocab // 3] = top
    check(sq, torch, x)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("vocab,far", [(32000, 7.15), (131072, 11.15)])
def test_one_logit_and_many_alike_in_16_bits(sq, torch, vocab, far, dtype):  # noqa: F811
    top = torch.tensor([0.0, 5.3, -2.7, 1e-3, 17.9, -60.1])
    x = (top - far)[:, None].repeat(1, vocab)
    x[:, 7] = top
    check(sq, torch, x.to(getattr(torch, dtype)))


def test_few_values(sq, torch):  # noqa: F811
    # two and three values in turn, so that pairs and rows of pairs err alike
    g = torch.Generator().manual_seed(1)
    for k in range(12):
        values = -11 * torch.rand(2 + k % 3, generator=g)
        x = values[torch.arange(131072) % len(values)][None].contiguous()
        x[0, 5] = 1.0
        check(sq, torch, x)


@pytest.mark.parametrize("dtype", TYPES)
def test_where_the_terms_change_their_scale(sq, torch, dtype):  # noqa: F811
    # largest logits of +-48 and next to it, many alike below them, rising rows across it
    tops = torch.tensor([47.75, 48.0, 48.25, 49.5, -47.75, -48.0, -48.25, -60.0, 96.0, -300.0])
    for far in (0.25, 9.0, 11.25, 13.5, 20.0):
        x = (tops - far)[:, None].repeat(1, 40001)
        x[:, 40000] = tops
        check(sq, torch, x.to(getattr(torch, dtype)))
    for lo, hi in ((-60.0, 60.0), (40.0, 56.0), (-55.0, -40.0)):
        check(sq, torch, torch.linspace(lo, hi, 3001).to(getattr(torch, dtype))[None].contiguous())


@pytest.mark.parametrize("vocab", [300, 5000, 70001])
def test_large_logits(sq, torch, vocab):  # noqa: F811
    # past 2^20, where fp32 is coarse and the differences are exact; rising and falling rows
    g = torch.Generator().manual_seed(vocab)
    rows = []
    for top in (1048575.9375, 1048576.0, 1048583.5, -1048583.5, -1048570.5, 3.0e6, -3.0e6, 1.5e9, -2.0e30, 3.3e38, -3.3e38):
        step = np.spacing(np.float32(abs(top)))
        rows.append((np.float64(top) - step * torch.randint(0, 60, (vocab,), generator=g).double().numpy()).astype(np.float32))
    x = torch.from_numpy(np.stack(rows))
    x[:3, ::7] = -3.4028234663852886e38
    x[2, ::11] = float("-inf")
    x = x.clamp(max=3.4028234663852886e38)
    check(sq, torch, x)
    check(sq, torch, x.sort(1).values)
    check(sq, torch, x.sort(1, descending=True).values)


@pytest.mark.parametrize("vocab", [515, 40000])
def test_sums_whose_largest_logit_comes_late(sq, torch, vocab):  # noqa: F811
    # every logit raises the largest: a sum is scaled again and again, over all magnitudes
    for lo, hi in ((-30.0, 3.0), (-2.0, 0.0), (-3e6, 40.0), (1.0e6, 1.06e6), (-1.0485762e6, -1.0485756e6), (-1e38, 2.0)):
        check(sq, torch, torch.linspace(lo, hi, vocab, dtype=torch.float64).float()[None].contiguous())
    x = torch.full((3, vocab), -3.4028234663852886e38)
    x[0, -1], x[1, vocab // 2], x[2, -2:] = 0.0, -5.0, 1e-30
    check(sq, torch, x)
    x[:] = float("-inf")
    x[0, -1], x[1, 0] = -1e4, 2.0 ** 21
    check(sq, torch, x)
