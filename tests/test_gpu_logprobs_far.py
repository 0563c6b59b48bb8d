"""The gradient of rows whose log of the sum is too large for fp32 to hold the log of the
number of tokens in it, against the oracle with its own lse in 64 bits. Rows of nothing but
a type's lowest value, as a mask that bars every token leaves, are the plainest.

Bars: those of test_gpu_logprobs.py. p comes from x - m, which is exact or rounded to 2^-24
of itself, minus log S, rounded to 2^-24 of itself; both are at most |log p| here, so p errs
by no more than 2^-22 |log p| and the sums' 2^-21 of itself."""
import numpy as np
import pytest

from oracle import logprobs as olp
from test_gpu_logprobs import TINY, TYPES, UNIT, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def _rows(torch, vocab, dtype):
    dt = getattr(torch, dtype)
    low = torch.finfo(dt).min
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(12, vocab, generator=g)
    x[0] = low                                  # a mask of the lowest value over everything
    x[1] = low
    x[1, ::3] = -INF
    x[2] = -10000.0                             # a mask by addition
    x[3] -= 10000.0
    x[4] = x[4] * 300 + 20000                   # far up, spread
    x[5] = 30000.0
    x[6, : vocab // 2] = low                    # half masked: not far
    x[7] = x[7] * 2 + 1030                      # at the line
    x[8] = x[8] * 2 + 1000
    x[9] = low / 2
    x[9, vocab // 2] = low / 2 * 0.998
    x[10] = -INF
    x[10, 1] = 5000.0                           # one token left
    tokens = torch.randint(vocab, (12,), generator=g)
    tokens[9], tokens[10] = vocab // 2, 1
    tokens[3] = -1
    return x.to(dt), tokens


def _check(d, x, tokens, entropy, g, h, dtype):
    for t in range(x.shape[0]):
        xt, tok = x[t].double().numpy(), int(tokens[t])
        lse = olp.row(xt, tok, 0)[2]
        m = xt.max()
        log_s = np.log(np.exp(xt - m).sum())
        gt, ht, ent = float(g[t]), float(h[t]), float(entropy[t])
        # the oracle's formula with lse as m and log S, exact at any magnitude
        ref = olp.gradient(xt - m, tok, log_s, ent, gt, ht)
        assert abs(lse - (m + log_s)) <= 1e-9 * abs(lse)
        lp = xt - m - log_s
        with np.errstate(invalid="ignore"):
            p = np.exp(lp)
            size = np.where(p > 0, np.abs(lp), 0)
            part = p * (abs(gt if tok >= 0 else 0.0) + abs(ht) * (size + ent))
        bar = UNIT[dtype] * np.abs(ref) * 1.001 + TINY[dtype] + part * (2.0 ** -21 + 2.0 ** -22 * size)
        if abs(lse) < 1024:                     # the lse as it was kept, in fp32
            bar = bar + part * 2.0 ** -23 * abs(lse)
        assert np.all(np.abs(d[t] - ref) <= bar), (t, np.max(np.abs(d[t] - ref) - bar))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [7, 40, 1001, 3001, 70000])
def test_gradient_where_fp32_cannot_hold_the_lse(sq, torch, vocab, dtype):
    x, tokens = _rows(torch, vocab, dtype)
    gen = torch.Generator().manual_seed(3)
    g, h = torch.randn(12, generator=gen), torch.randn(12, generator=gen)
    dx, dt = x.cuda(), tokens.cuda()
    r = sq.token_logprobs(dx, dt)
    args = (r.lse, r.entropy, g.cuda(), h.cuda())
    d = sq.token_logprobs_backward(dx, dt, *args)
    _check(d.double().cpu().numpy(), x, tokens, r.entropy.cpu(), g, h, dtype)
    # a lone g and a lone h
    zero = torch.zeros(12)
    d2 = sq.token_logprobs_backward(dx, dt, r.lse, None, g.cuda())
    _check(d2.double().cpu().numpy(), x, tokens, zero, g, zero, dtype)
    # in place, and inside a larger buffer: the same bits
    wide = torch.full((12, vocab + 9), 7.0, dtype=x.dtype, device="cuda")
    y = wide[:, 3:3 + vocab]
    y.copy_(dx)
    sq.token_logprobs_backward(y, dt, *args, out=y)
    assert torch.equal(y, d) and (wide[:, :3] == 7.0).all() and (wide[:, 3 + vocab:] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_fully_masked_row_is_uniform(sq, torch, dtype):
    dt = getattr(torch, dtype)
    x = torch.full((2, 1000), torch.finfo(dt).min, dtype=dt, device="cuda")
    tokens = torch.tensor([3, 999], device="cuda")
    r = sq.token_logprobs(x, tokens)
    d = sq.token_logprobs_backward(x, tokens, r.lse, grad_logprob=torch.ones(2, device="cuda")).float()
    assert abs(d[0, 3].item() - 0.999) < 2 ** -8 and abs(d[0, 4].item() + 0.001) < 1e-5
    assert (d.sum(1).abs() < 5e-3).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_token_outside_an_empty_row(sq, torch, dtype):
    # with a gradient at its log probability NaN, as the log probability itself is; without, 0
    x = torch.full((2, 300), -INF, dtype=getattr(torch, dtype), device="cuda")
    tokens = torch.tensor([300, 5], device="cuda")
    one = torch.ones(2, device="cuda")
    r = sq.token_logprobs(x, tokens)
    assert np.isnan(r.logprob[0].item()) and r.logprob[1].item() == -INF
    d = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, one, one)
    assert d[0].isnan().all() and not d[1].any()
    d = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, None, one)
    assert not d.any()
