"""The operators past the sizes that one launch takes (2^21 rows, 32768 vectors), where
the ways of a product meet, and together as a user has them.

Bars: what a call gives for many rows equals what it gives for the same rows in
smaller calls, bit for bit, since a row's sums have the same order in both; products
against 64 bits as for other sizes. Eight columns add at most eight terms of at most 15
scales each, so partial sums stay within 15 sqrt(8) / 4.6 = 9.2 times the result's rms and
their roundings, 2^-24 of them, sum to at most 5e-6 of it: within the bars of
``_check_product``."""
import numpy as np
import pytest

from oracle import logprobs as olp
from oracle import q4 as oq4
from test_gpu_q4 import TYPES, _check_product, _random_q4, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu

EDGE = 1 << 21
ROWS = EDGE + 37


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
def test_quantise_and_dequantise_more_rows_than_a_launch(sq, torch, zeros, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    W = (torch.randn(ROWS, 8, device="cuda", generator=g) * 0.02).to(getattr(torch, dtype))
    q = sq.q4_quantize(W, 32, zeros=zeros)
    back = sq.q4_dequantize(q, W.dtype)
    for a, b in ((0, 1000), (EDGE - 500, EDGE + 1), (EDGE, ROWS), (ROWS - 3, ROWS)):
        part = sq.q4_quantize(W[a:b].contiguous(), 32, zeros=zeros)
        assert torch.equal(part.codes, q.codes[a:b]) and torch.equal(part.scale, q.scale[a:b])
        assert not zeros or torch.equal(part.zero, q.zero[a:b])
        assert torch.equal(sq.q4_dequantize(part, W.dtype), back[a:b])
    a = EDGE - 20
    codes, scale, zero = oq4.quantize(W[a:a + 50].double().cpu().numpy(), 32, zeros)
    assert np.array_equal(oq4.pack(codes).view(np.int32), q.codes[a:a + 50].cpu().numpy())
    assert np.array_equal(scale, q.scale[a:a + 50].cpu().numpy())
    assert not zeros or np.array_equal(zero, q.zero[a:a + 50].cpu().numpy())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 4, 20])
def test_product_of_more_rows_than_a_launch(sq, torch, nvec, dtype):
    rng = np.random.default_rng(nvec)
    q, W = _random_q4(sq, torch, rng, ROWS, 8, 32, True)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, 8)).astype(np.float32)).to(getattr(torch, dtype))
    y = sq.q4_gemv(q, x.cuda(), torch.float32)
    for a, b in ((0, 300), (EDGE - 300, ROWS)):
        _check_product(y[:, a:b], x.double().numpy() @ W[a:b].T, "float32")
    exact = torch.from_numpy(W).cuda() @ x.double().cuda().t()
    assert ((y.double() - exact.t()).norm() / exact.norm()).item() <= 1e-6


@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_more_vectors_than_a_launch(sq, torch, dtype):
    rng = np.random.default_rng(4)
    n = 32768 + 45
    q, W = _random_q4(sq, torch, rng, 40, 72, 32, True)
    x = torch.from_numpy(rng.normal(0, 1, (n, 72)).astype(np.float32)).to(getattr(torch, dtype))
    y = sq.q4_gemv(q, x.cuda(), torch.float32)
    _check_product(y, x.double().numpy() @ W.T, "float32")


@pytest.mark.parametrize("rows,cols,nvec,dtype", [
    (77, 1032, 4, "float32"), (77, 1032, 5, "float32"), (77, 1032, 7, "float32"), (77, 1032, 8, "float32"),
    (77, 1032, 9, "float32"), (4104, 4096, 4, "float32"), (4104, 4096, 5, "float32"),
    (4104, 4096, 2, "bfloat16"), (4104, 4096, 3, "bfloat16"), (8192, 1032, 2, "float16"),
    (8192, 1032, 16, "float16"), (8192, 1032, 17, "float16"), (16384, 520, 1, "bfloat16")])
def test_products_where_the_ways_meet(sq, torch, rows, cols, nvec, dtype):
    rng = np.random.default_rng(rows + nvec)
    q, W = _random_q4(sq, torch, rng, rows, cols, 128, True)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(getattr(torch, dtype))
    _check_product(sq.q4_gemv(q, x.cuda(), torch.float32), x.double().numpy() @ W.T, "float32")


@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_of_more_rows_than_a_launch(sq, torch, dtype):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = (torch.randn(ROWS, 5, device="cuda", generator=g) * 3).to(getattr(torch, dtype))
    tokens = torch.randint(-1, 5, (ROWS,), device="cuda", generator=g)
    r = sq.token_logprobs(x, tokens, top=2)
    one = torch.ones(ROWS, device="cuda")
    grad = sq.token_logprobs_backward(x, tokens, r.lse, r.entropy, one, one)
    for a, b in ((0, 100), (EDGE - 100, EDGE + 1), (EDGE, ROWS)):
        s = sq.token_logprobs(x[a:b].contiguous(), tokens[a:b].contiguous(), top=2)
        for k in ("logprob", "entropy", "lse", "top_token", "top_logprob"):
            assert torch.equal(getattr(r, k)[a:b], getattr(s, k)), k
        assert torch.equal(grad[a:b], sq.token_logprobs_backward(
            x[a:b].contiguous(), tokens[a:b].contiguous(), s.lse, s.entropy, one[a:b].contiguous(),
            one[a:b].contiguous()))
    for t in (EDGE - 1, EDGE, ROWS - 1):
        lp, entropy, lse, alts = olp.row(x[t].double().cpu().numpy(), int(tokens[t]), 2)
        got = [v[t].item() for v in (r.logprob, r.entropy, r.lse)]
        assert np.allclose(got, [lp, entropy, lse], rtol=1e-6, atol=4e-6)
        assert r.top_token[t].tolist() == [v for v, _ in alts]


def test_streams_of_another_device_are_refused(sq):
    class Elsewhere:
        cuda_stream = 0

        class device:
            index = 1
    import torch as t
    W = t.zeros(1, 32, device="cuda")
    with pytest.raises(ValueError, match="stream"):
        sq.q4_quantize(W, 32, stream=Elsewhere())


def test_scoring_runs_the_operators_together(sq, torch):
    from paper_2609_38477_amd import scoring
    W, h, tokens = scoring.sample(1000, 256, 70)
    res = scoring.study(W, h, tokens, 64, zeros=True)
    base, q4, seed = (res["heads"][k] for k in ("original", "q4", "seed"))
    # against 64 bits: the log likelihood of the same tokens
    z = h.double() @ W.double().t()
    nll = (torch.logsumexp(z, 1) - z.gather(1, tokens[:, None]).squeeze(1)).mean().item()
    assert abs(base["nll"] - nll) < 1e-5 * (1 + nll)
    q = sq.q4_quantize(W, 64, zeros=True)
    z = h.double() @ sq.q4_dequantize(q).double().t()
    nll = (torch.logsumexp(z, 1) - z.gather(1, tokens[:, None]).squeeze(1)).mean().item()
    assert abs(q4["nll"] - nll) < 1e-5 * (1 + nll)
    assert q4["bits_per_weight"] == 4 + 24 / 64 and abs(seed["bits_per_weight"] - 4) < 0.1
    # tokens were drawn from the original's softmax: it is the likeliest of the three
    assert base["perplexity"] < min(q4["perplexity"], seed["perplexity"]) < 1000
    assert base["same_first_token"] == 1.0 and q4["same_first_token"] > 0.5
    # the gradient of the log likelihood: sum_r W_rj^2 mean_t (p_tr - 1[r = tok])^2
    z = h.double() @ W.double().t()
    g = torch.softmax(z, 1)
    g[torch.arange(70, device="cuda"), tokens] -= 1
    rho = ((W.double() ** 2) * (g ** 2).mean(0)[:, None]).sum(0).cpu().numpy()
    assert np.allclose(scoring.measured_rho(W, h @ W.t(), tokens), rho, rtol=1e-4)
    token, logprob = scoring.next_token(q, h[0])
    z = (h[:1].double() @ sq.q4_dequantize(q).double().t()).log_softmax(1)[0]
    assert abs(z[token].cpu().numpy() - logprob.cpu().numpy()).max() < 1e-4
    faults = res["q4_faults"]
    assert [f["N_flip"] for f in faults[:2]] == [1, 1] and faults[4]["N_flip"] == 64
    assert all(0 < f["N_flip"] <= 64 for f in faults[2:4])
