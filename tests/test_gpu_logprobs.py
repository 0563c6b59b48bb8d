"""Log probabilities of given tokens, entropy, top alternatives and their gradient on
the GPU against the oracle.

Bars, absolute: log probabilities 1e-6 + 2^-22 |value| and lse the same (the
log of the sum: terms within 2^-22, sums of non-negative terms within 2^-21); entropy
2e-6 (1 + value), its two parts being such sums. Tokens equal. The gradient: the
type's half unit of the value, plus 2^-21 + 2^-22 |log p| of p (|g| + |h| (|log p| +
entropy)), from the rounding of x - lse and of the exponential."""
import numpy as np
import pytest

from oracle import logprobs as olp

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")
UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 1e-38, "float16": 2.0 ** -25, "bfloat16": 1e-38}
INF = float("inf")


@pytest.fixture(scope="module")
def sq():
    import paper_2609_38477_amd as sq
    sq.lib()
    return sq


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _near(got, ref, bar):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    same = (got == ref) | np.isnan(ref)
    with np.errstate(invalid="ignore"):
        assert np.all(same | (np.abs(got - ref) <= bar(np.abs(ref)))), np.nanmax(np.abs(got - ref))


def _check(sq, torch, x, tokens, top):
    """Every output of one call against the oracle, row by row; returns the call's result."""
    r = sq.token_logprobs(x, tokens, top=top)
    rows = [olp.row(x[t].double().cpu().numpy(), int(tokens[t]), top) for t in range(x.shape[0])]
    _near(r.logprob.cpu(), [v[0] for v in rows], lambda a: 1e-6 + a * 2.0 ** -22)
    _near(r.entropy.cpu(), [v[1] for v in rows], lambda a: 2e-6 * (1 + a))
    _near(r.lse.cpu(), [v[2] for v in rows], lambda a: 1e-6 + a * 2.0 ** -22)
    if top:
        assert r.top_token.shape == (x.shape[0], top)
        assert r.top_token.cpu().tolist() == [[t for t, _ in v[3]] for v in rows]
        _near(r.top_logprob.cpu(), [[p for _, p in v[3]] for v in rows],
              lambda a: 1e-6 + a * 2.0 ** -22)
    else:
        assert r.top_token is None and r.top_logprob is None
    return r


def _logits(torch, rows, vocab, dtype, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab + pad, generator=g) * 4.0
    tokens = torch.randint(vocab, (rows,), generator=g)
    return x.to(getattr(torch, dtype)).cuda()[:, :vocab], tokens.cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 31), (5, 33), (4, 257), (3, 1000),
                                        (2, 4099), (1, 32003), (7, 8192)])
def test_rows_of_every_length(sq, torch, rows, vocab, top, dtype):
    x, tokens = _logits(torch, rows, vocab, dtype, rows * vocab + top)
    _check(sq, torch, x, tokens, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 131072), (2, 262147), (300, 2048), (1100, 640)])
def test_long_rows_and_many_rows(sq, torch, rows, vocab, dtype):
    x, tokens = _logits(torch, rows, vocab, dtype, vocab)
    x = x.clone()
    few = min(rows, 4)
    r = sq.token_logprobs(x, tokens, top=20)
    some = sq.token_logprobs(x[:few].contiguous(), tokens[:few].contiguous(), top=20)
    last = _check(sq, torch, x[rows - few:].contiguous(), tokens[rows - few:].contiguous(), 20)
    # a row's result does not depend on the rows beside it, but for the order of its sums
    for a, b, c in zip(r.__dict__.values(), some.__dict__.values(), last.__dict__.values()):
        if a.dtype == torch.int64:
            assert torch.equal(a[:few], b) and torch.equal(a[rows - few:], c)
        else:
            assert torch.allclose(a[:few], b, atol=3e-6, rtol=1e-6)
            assert torch.allclose(a[rows - few:], c, atol=3e-6, rtol=1e-6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 3001, 70000])
def test_masks_and_values_that_are_not_finite(sq, torch, vocab, dtype):
    dt = getattr(torch, dtype)
    low = torch.finfo(dt).min
    x, tokens = _logits(torch, 16, vocab, dtype, vocab)
    x = x.clone()
    x[0] = -INF                                # nothing left
    x[1] = -INF
    x[1, vocab - 1] = 3.0                      # one token left
    x[2] = -INF
    x[2, ::7] = 1.5                            # ties among a few
    x[3] = low                                 # the type's lowest value everywhere: uniform
    x[4] = low
    x[4, 3] = 1.0
    x[5, vocab // 2] = INF
    x[6, vocab // 3] = float("nan")
    x[7] = 0.0                                 # all equal
    x[7, ::2] = -0.0                           # -0 ties with 0
    x[8] = -INF
    x[8, 5] = low
    x[9] = torch.finfo(dt).max / 2             # large and equal
    x[10, : vocab // 2] = -INF                 # half masked
    x[11] = -INF
    x[11, 0] = float("nan")                    # a NaN among masked ones
    x[12, 0] = INF
    x[12, 1] = -INF
    tokens[10] = 1                             # a masked token
    tokens[13] = -1
    tokens[14] = vocab                         # outside
    tokens[15] = -100
    tokens[5], tokens[6] = vocab // 2, -1
    r = _check(sq, torch, x, tokens, 12)
    assert r.top_token[0].tolist() == [-1] * 12 and r.logprob[0] == -INF and r.entropy[0] == 0
    assert r.top_token[7].tolist() == list(range(12))
    assert r.top_token[6].tolist() == [-1] * 12 and r.logprob[6] == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_alternatives_wherever_they_lie(sq, torch, dtype):
    # rising, falling, and the largest ones side by side or far apart; ties at the cut
    vocab = 9001
    x = torch.zeros(8, vocab)
    ramp = torch.arange(vocab) / 64.0
    x[0], x[1] = ramp, ramp.flip(0)
    x[2, 4000:4040] = torch.arange(40) / 8.0
    x[3, torch.arange(0, 32) * 256] = torch.arange(32) / 4.0 + 1
    x[4, -32:] = 5.0
    x[5] = torch.arange(vocab) % 13
    x[6, :64] = 2.0
    x[7, 8::1024] = 4.0
    x[7, 9::1024] = 4.0
    tokens = torch.arange(8).cuda() * 1000
    for top in (1, 2, 20, 32):
        _check(sq, torch, x.to(getattr(torch, dtype)).cuda(), tokens, top)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_anywhere_and_on_another_stream(sq, torch, dtype):
    vocab = 1999
    x, tokens = _logits(torch, 6, vocab, dtype, 3, pad=11)
    wide = torch.full((6, vocab + 11), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 5:5 + vocab] = x
    view = wide[:, 5:5 + vocab]                # odd start, odd stride, NaN around
    ref = _check(sq, torch, view, tokens, 7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for r in (sq.token_logprobs(x.contiguous(), tokens, top=7),
              sq.token_logprobs(x.t().contiguous().t(), tokens, top=7),
              sq.token_logprobs(view, tokens, top=7, stream=s)):
        s.synchronize()
        assert torch.equal(r.top_token, ref.top_token)
        assert torch.allclose(r.logprob, ref.logprob, atol=3e-6, rtol=1e-6)
    again = sq.token_logprobs(view, tokens, top=7)
    for a, b in zip(ref.__dict__.values(), again.__dict__.values()):
        assert torch.equal(a, b)               # the same bits from run to run
    none = sq.token_logprobs(view)
    assert none.logprob is None and torch.equal(none.lse, ref.lse)
    empty = sq.token_logprobs(x[:0], tokens[:0], top=3)
    assert empty.logprob.shape == (0,) and empty.top_token.shape == (0, 3)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 32000, "float32"), (1, 200000, "bfloat16"),
                                              (64, 5000, "float16")])
def test_in_a_graph(sq, torch, rows, vocab, dtype):
    xs = [_logits(torch, rows, vocab, dtype, k) for k in range(4)]
    refs = [sq.token_logprobs(x, t, top=4) for x, t in xs]
    x, tokens = xs[0][0].clone(), xs[0][1].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sq.token_logprobs(x, tokens, top=4)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = sq.token_logprobs(x, tokens, top=4)
        d = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, r.logprob, r.entropy)
    for (v, t), ref in zip(xs, refs):
        x.copy_(v)
        tokens.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(r.__dict__.values(), ref.__dict__.values()):
            assert torch.equal(a, b)
        assert torch.equal(d, sq.token_logprobs_backward(v, t, ref.lse, ref.entropy, ref.logprob,
                                                         ref.entropy))


# ---------------------------------------------------------------- gradient

def _check_gradient(sq, torch, x, tokens, g, h, dtype):
    r = sq.token_logprobs(x, tokens)
    d = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, g, h)
    assert d.dtype == x.dtype and d.shape == x.shape
    for t in range(x.shape[0]):
        gt = 0.0 if g is None else float(g[t])
        ht = 0.0 if h is None else float(h[t])
        lse, ent = float(r.lse[t]), float(r.entropy[t])
        xt = x[t].double().cpu().numpy()
        tok = int(tokens[t]) if g is not None else -1
        ref = olp.gradient(xt, tok, lse, ent, gt, ht)
        got = d[t].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        with np.errstate(invalid="ignore", over="ignore"):
            lp = xt - lse
            p = np.exp(lp)
            part = p * (abs(gt) + abs(ht) * (np.where(p > 0, np.abs(lp), 0) + ent))
            bar = (UNIT[dtype] * np.abs(ref) * 1.001 + TINY[dtype] +
                   part * (2.0 ** -21 + 2.0 ** -22 * np.where(p > 0, np.abs(lp), 0)))
            bar = np.where(np.isfinite(bar), bar, 0)
            assert np.all(np.isnan(ref) | (np.abs(got - ref) <= bar)), (t, np.nanmax(np.abs(got - ref) - bar))
    return d


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["logprob", "entropy", "both"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (3, 7, 2), (5, 1000, 0), (2, 4099, 3),
                                            (1, 65537, 0), (4, 2048, 8)])
def test_gradient_matches_the_formula(sq, torch, rows, vocab, pad, which, dtype):
    x, tokens = _logits(torch, rows, vocab, dtype, vocab, pad)
    gen = torch.Generator().manual_seed(7)
    g = torch.randn(rows, generator=gen).cuda() if which != "entropy" else None
    h = torch.randn(rows, generator=gen).cuda() if which != "logprob" else None
    if vocab > 1:
        x = x.clone()
        x[:, ::5] = -INF
        x[0, 1] = 2.0
    _check_gradient(sq, torch, x, tokens, g, h, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_of_rows_without_a_distribution(sq, torch, dtype):
    x, tokens = _logits(torch, 6, 700, dtype, 1)
    x = x.clone()
    x[0] = -INF
    x[1, 5] = float("nan")
    x[2, 5] = INF
    tokens[3] = -1
    tokens[4] = 700
    one = torch.ones(6, device="cuda")
    d = _check_gradient(sq, torch, x, tokens, one, one, dtype)
    assert not d[0].any() and d[1].isnan().all() and d[2].isnan().all() and d[4].isnan().all()
    d = _check_gradient(sq, torch, x, tokens, one, None, dtype)
    assert not d[3].any()                              # no token asked: no gradient


def test_gradient_against_differences(sq, torch):
    # central differences of the oracle's value at the GPU's own gradient
    x, tokens = _logits(torch, 3, 23, "float32", 2)
    g, h = torch.tensor([1.0, -0.5, 0.3]).cuda(), torch.tensor([0.2, 0.0, -1.0]).cuda()
    r = sq.token_logprobs(x, tokens)
    d = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, g, h).double().cpu().numpy()
    xs, e = x.double().cpu().numpy(), 1e-5
    for t in range(3):
        for v in range(23):
            up, dn = xs[t].copy(), xs[t].copy()
            up[v] += e
            dn[v] -= e
            a, b = olp.row(up, int(tokens[t]), 0), olp.row(dn, int(tokens[t]), 0)
            num = (float(g[t]) * (a[0] - b[0]) + float(h[t]) * (a[1] - b[1])) / (2 * e)
            # 2^-21 + 2^-22 |log p| of at most p (1 + |log p| + entropy) < 4, and 1e-9
            # from the differences
            assert abs(num - d[t, v]) < 1e-5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [0, 5])
def test_gradient_in_place_and_inside_a_larger_buffer(sq, torch, pad, dtype):
    x, tokens = _logits(torch, 9, 3001, dtype, 4, pad)
    g = torch.linspace(-1, 1, 9).cuda()
    r = sq.token_logprobs(x, tokens)
    ref = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, g, g)
    wide = torch.full((9, 3001 + 14), 7.0, dtype=x.dtype, device="cuda")
    sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, g, g, out=wide[:, 3:3004])
    assert torch.equal(wide[:, 3:3004], ref)
    assert (wide[:, :3] == 7.0).all() and (wide[:, 3004:] == 7.0).all()
    base = torch.full((9, 3001 + pad), 7.0, dtype=x.dtype, device="cuda")
    y = base[:, :3001]
    y.copy_(x)
    got = sq.token_logprobs_backward(y, tokens, r.lse, r.entropy, g, g, out=y)
    assert got.data_ptr() == y.data_ptr() and torch.equal(y, ref)
    assert (base[:, 3001:] == 7.0).all()


def test_offsets_past_32_bits(sq, torch):
    # 2^32 logits and more in bf16: the last row's sums and gradient
    rows, vocab = 33000, 131075
    x = torch.full((rows, vocab), -1.0, dtype=torch.bfloat16, device="cuda")
    x[-1, -1] = 9.0
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    tokens[-1] = vocab - 1
    r = sq.token_logprobs(x, tokens, top=2)
    lse = np.log(np.exp(10.0) + vocab - 1) - 1.0
    assert abs(float(r.lse[-1]) - lse) < 4e-6 and r.top_token[-1].tolist() == [vocab - 1, 0]
    assert abs(float(r.lse[0]) - (np.log(vocab) - 1.0)) < 4e-6 and r.top_token[0].tolist() == [0, 1]
    g = torch.ones(rows, device="cuda")
    sq.token_logprobs_backward(x, tokens, r.lse, None, g, None, out=x)
    p = np.exp(9.0 - lse)
    assert abs(float(x[-1, -1]) - (1 - p)) < 2.0 ** -9
    assert abs(float(x[-1, 0]) + np.exp(-1.0 - lse)) < 1e-7
    assert abs(float(x[0, 0]) - (1 - 1 / vocab)) < 2.0 ** -8


def test_helpers_refuse_wrong_tensors(sq, torch):
    x = torch.zeros(4, 10, device="cuda")
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    for bad in (tok[:3], tok.int(), tok.cpu(), tok[:, None]):
        with pytest.raises(ValueError):
            sq.token_logprobs(x, bad)
    for top in (-1, 33):
        with pytest.raises(ValueError):
            sq.token_logprobs(x, tok, top=top)
    with pytest.raises(ValueError):
        sq.token_logprobs(x[:, :0], tok)
    for kw in (dict(lse=f[:2]), dict(lse=f.double()), dict(lse=f, grad_logprob=f[:1]),
               dict(lse=f, grad_entropy=f), dict(lse=f), dict(lse=f, grad_logprob=f, out=f),
               dict(lse=f, grad_logprob=f, out=x.half()), dict(lse=f, grad_logprob=f, out=x.t())):
        with pytest.raises(ValueError):
            sq.token_logprobs_backward(x, tok, **kw)
