"""Log probabilities by the workgroups of four waves that many rows of middle length take,
and the slow selection of alternatives, which a row takes whose largest elements lie in the
vectors of a few threads, against 64 bits.

A thread of NT owns the vectors v (16 bytes) with v % NT its index, and 64 groups of
neighbouring threads bound the alternatives from below; with fewer groups of large elements
than alternatives the bound is an ordinary element and every large one is found. Bars: those
of test_gpu_logprobs.py."""
import numpy as np
import pytest

from oracle import logprobs as olp
from test_gpu_logprobs import TYPES, _near, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")
KEPT = {64: 512, 256: 1024, 512: 1024}     # elements that a workgroup keeps


def _check_rows(torch, r, x, tokens, top, odd=()):
    """r against 64 bits: the rows of `odd` by the oracle, the others (all finite) by torch."""
    plain = torch.ones(x.shape[0], dtype=torch.bool)
    plain[list(odd)] = False
    xd = x.double()
    lse = torch.logsumexp(xd, 1)
    lp = xd.gather(1, tokens.clamp(0, x.shape[1] - 1)[:, None]).squeeze(1) - lse
    logp = xd - lse[:, None]
    ent = -(logp.exp() * logp).sum(1)
    bar = lambda a: 1e-6 + a * 2.0 ** -22   # noqa: E731
    _near(r.lse.cpu()[plain], lse.cpu()[plain], bar)
    _near(r.logprob.cpu()[plain], torch.where(tokens < 0, 0.0, lp).cpu()[plain], bar)
    _near(r.entropy.cpu()[plain], ent.cpu()[plain], lambda a: 2e-6 * (1 + a))
    if top:
        v, i = torch.sort(xd, dim=1, descending=True, stable=True)
        assert torch.equal(r.top_token.cpu()[plain], i[:, :top].cpu()[plain])
        _near(r.top_logprob.cpu()[plain], (v[:, :top] - lse[:, None]).cpu()[plain], bar)
    for t in odd:
        want = olp.row(xd[t].cpu().numpy(), int(tokens[t]), top)
        _near([r.logprob[t].item(), r.lse[t].item()], [want[0], want[2]], bar)
        _near([r.entropy[t].item()], [want[1]], lambda a: 2e-6 * (1 + a))
        if top:
            assert r.top_token[t].tolist() == [v for v, _ in want[3]]
            _near(r.top_logprob[t].cpu(), [p for _, p in want[3]], bar)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [0, 1, 20, 32])
@pytest.mark.parametrize("rows,vocab", [(600, 4100), (1030, 9001)])
def test_many_rows_of_middle_length(sq, torch, rows, vocab, top, dtype):
    g = torch.Generator(device="cuda").manual_seed(vocab + top)
    dt = getattr(torch, dtype)
    x = (torch.randn(rows, vocab + 3, device="cuda", generator=g) * 4).to(dt)[:, :vocab]
    tokens = torch.randint(vocab, (rows,), device="cuda", generator=g)
    low = torch.finfo(dt).min
    x[0] = -INF
    x[1, : vocab - 3] = -INF                       # three left, two of them after the last vector
    x[2, 17] = float("nan")
    x[3, vocab - 1] = INF
    x[4] = low
    x[5] = -INF
    x[5, ::513] = 2.0                              # ties among a few
    x[6, : vocab // 2] = -INF
    x[10] = 0.0                                    # all equal
    x[11] = (torch.arange(vocab, device="cuda") % 13).to(dt)
    x[12] = (torch.arange(vocab, device="cuda") / 64.0).to(dt)
    tokens[7], tokens[8], tokens[6] = -1, vocab, 3
    odd = (0, 1, 2, 3, 4, 5, 6, 8, rows - 1)
    _check_rows(torch, sq.token_logprobs(x, tokens, top=top), x, tokens, top, odd)


def _found(x, per_vector, threads, top):
    """Elements of one workgroup's part of a row that reach its bound."""
    n = x.size // (per_vector * threads) * (per_vector * threads)
    best = x[:n].reshape(-1, threads, per_vector).max(axis=(0, 2))
    groups = np.sort(best.reshape(64, -1).max(axis=1))[::-1]
    return int((x >= groups[top - 1]).sum())


@pytest.mark.parametrize("rows,vocab,dtype,threads,segments", [
    (3, 2048, "bfloat16", 64, 1), (3, 2051, "float16", 64, 1), (1030, 4096, "float32", 64, 1),
    (600, 4100, "float32", 256, 1), (600, 4103, "bfloat16", 256, 1), (520, 20000, "float16", 256, 1),
    (2, 33003, "float32", 512, 1), (2, 66005, "bfloat16", 512, 1),
    (2, 131072, "float32", 512, 8), (3, 131079, "bfloat16", 512, 4)])
@pytest.mark.parametrize("ties", [False, True])
def test_largest_elements_in_the_vectors_of_a_few_threads(sq, torch, rows, vocab, dtype, threads,
                                                          segments, ties):
    top, per_vector = 32, 4 if dtype == "float32" else 8
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, device="cuda", generator=g)
    large = (torch.arange(vocab, device="cuda") // per_vector) % threads < 20 * (threads // 64)
    lift = torch.randint(8, (rows, vocab), device="cuda", generator=g) * 1.0 if ties else \
        torch.rand(rows, vocab, device="cuda", generator=g) * 9.0
    x = torch.where(large, 10.0 + lift, x).to(getattr(torch, dtype))
    x[-1] = torch.randn(vocab, device="cuda", generator=g).to(x.dtype)       # an ordinary row beside them
    # the case is what it is for: more is found than kept, in every segment
    vectors = -(-(vocab // per_vector) // segments) * per_vector
    for s in range(segments):
        part = x[0, s * vectors:(s + 1) * vectors].double().cpu().numpy()
        assert _found(part, per_vector, threads, top) > KEPT[threads]
    tokens = torch.randint(vocab, (rows,), device="cuda", generator=g)
    _check_rows(torch, sq.token_logprobs(x, tokens, top=top), x, tokens, top)
    _check_rows(torch, sq.token_logprobs(x, tokens, top=21), x, tokens, 21)
