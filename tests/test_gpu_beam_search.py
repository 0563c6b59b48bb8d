"""Beam search over a head and the microscaled head's figures: the selection, the
reordering and the products together, as a decoder uses them.

Bars: with as many beams as there are prefixes the search is exhaustive, so its best
sequences are those of all sequences' log probabilities in fp64; a step's total errs by
2e-7 and a rounding to fp32, 2^-24 of at most 32, so three steps by 8e-6, and sequences are
compared where their neighbours lie further apart."""
import itertools

import numpy as np
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def markov(torch, vocab, seed):  # noqa: F811
    """Logits of the next token from the last two, the state being the one before last."""
    g = torch.Generator().manual_seed(seed)
    table = (2 * torch.randn(vocab, vocab, vocab, generator=g)).cuda()

    def step(tokens, states):
        return table[states[0].view(-1), tokens].contiguous(), [tokens.unsqueeze(1)]
    return table, step


@pytest.mark.parametrize("eos", [-1, 2])
def test_an_exhaustive_search_finds_the_best_sequences(sq, torch, eos):  # noqa: F811
    from paper_2609_38477_amd import scoring
    vocab, length, beams, batch = 5, 3, 30, 4
    table, step = markov(torch, vocab, 7)
    first = torch.randint(vocab, (batch,)).cuda()
    before = torch.randint(vocab, (batch, 1)).cuda()
    found, score = scoring.beam_search(step, [before], first, beams, length, eos=eos, pad=1)
    logp = torch.log_softmax(table.double(), 2).cpu().numpy()
    for i in range(batch):
        every = {}
        for seq in itertools.product(range(vocab), repeat=length):
            a, b, total, out, done = int(before[i, 0]), int(first[i]), 0.0, [], False
            for v in seq:
                if done:
                    out.append(1)
                    continue
                total += logp[a, b, v]
                a, b, done = b, v, v == eos
                out.append(v)
            every[tuple(out)] = total
        want = sorted(every.items(), key=lambda e: -e[1])[:beams + 1]
        for r in range(beams):
            assert abs(score[i, r].item() - want[r][1]) < 8e-6
            near = [want[k][1] for k in (r - 1, r + 1) if 0 <= k < len(want)]
            if all(abs(v - want[r][1]) > 2e-5 for v in near):
                assert tuple(found[i, r].tolist()) == want[r][0]


def test_fewer_continuations_than_beams(sq, torch):  # noqa: F811
    from paper_2609_38477_amd import scoring
    _, step = markov(torch, 3, 1)
    zero = torch.zeros(2, dtype=torch.int64).cuda()
    found, score = scoring.beam_search(step, [zero.unsqueeze(1)], zero, 8, 1)
    assert (found[:, 3:] == -1).all() and (score[:, 3:] == float("-inf")).all()
    assert found[0, :3, 0].sort().values.tolist() == [0, 1, 2]
    assert torch.allclose(score[:, :3].exp().sum(1), torch.ones(2).cuda(), atol=1e-5)


def test_one_beam_is_the_likeliest_token_each_time(sq, torch):  # noqa: F811
    from paper_2609_38477_amd import scoring
    W, h, _ = scoring.sample(600, 128, 9)
    q = sq.mx4_quantize(W)
    found, score = scoring.continuations(lambda x: sq.mx4_gemv(q, x), W, h, 1, 4)
    first = sq.token_logprobs(sq.mx4_gemv(q, h), top=1)
    assert torch.equal(found[:, 0, 0], first.top_token[:, 0])
    four, best = scoring.continuations(lambda x: sq.mx4_gemv(q, x), W, h, 16, 4)
    assert found.shape == (9, 1, 4) and four.shape == (9, 16, 4)
    assert (best[:, 0] >= score[:, 0] - 1e-4).all() and (best[:, :-1] >= best[:, 1:]).all()


def test_the_study_reports_every_form(sq, torch):  # noqa: F811
    from paper_2609_38477_amd import scoring
    W, h, tokens = scoring.sample(600, 128, 40)
    r = scoring.study(W, h, tokens, 64, beams=3, length=4)
    heads = r["heads"]
    assert set(heads) == {"original", "q4", "seed", "mx4", "mx4_coded"}
    assert heads["mx4"]["bits_per_weight"] == 4.25
    exact = sq.mx4_dequantize(sq.mx4_quantize(W)).double()
    z = torch.log_softmax(h.double() @ exact.t(), 1).gather(1, tokens[:, None])
    assert abs(heads["mx4"]["nll"] + z.mean().item()) < 1e-5
    coded = sq.mx4_dequantize(sq.mx4_quantize(h)).double()
    z = torch.log_softmax(coded @ exact.t(), 1).gather(1, tokens[:, None])
    assert abs(heads["mx4_coded"]["nll"] + z.mean().item()) < 1e-5
    assert np.isfinite(list(r["beam_search"]["logprob"].values())).all()
