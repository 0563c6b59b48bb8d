"""The operators of seedq_ops.h without a GPU: exported symbols, argument errors
(reported before anything touches a GPU), the helpers' refusals, and the oracle's
own definitions against values worked out by hand."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import logprobs as olp
from oracle import q4 as oq4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "seedq_ops.h")
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -6


@pytest.fixture(scope="module")
def sq():
    import paper_2609_38477_amd as sq
    if not os.path.exists(sq.LIB_PATH):
        from paper_2609_38477_amd import build
        build.build()
    return sq


@pytest.fixture(scope="module")
def L(sq):
    return sq.ops.lib()


def test_every_declared_symbol_is_exported_and_wrapped(sq):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(seedq_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 8
    raw = ctypes.CDLL(sq.LIB_PATH)
    for n in names:
        assert hasattr(raw, n) and hasattr(sq, n), n


def test_row_words(sq):
    for c in (8, 24, 32, 40, 2056, 4096):
        assert sq.seedq_q4_row_words(c) == oq4.row_words(c)
    for c in (0, -8, 7, 12):
        assert sq.seedq_q4_row_words(c) == 0


def test_quantize_and_dequantize_argument_errors(L):
    def quantize(W=256, type=0, ldw=64, rows=4, cols=64, group=32, codes=256, scale=256, zero=None):
        return L.seedq_q4_quantize(W, type, ldw, rows, cols, group, codes, scale, zero, None)

    def dequantize(codes=256, scale=256, zero=None, rows=4, cols=64, group=32, W=256, type=0, ldw=64):
        return L.seedq_q4_dequantize(codes, scale, zero, rows, cols, group, W, type, ldw, None)

    for f in (quantize, dequantize):
        for bad in (dict(W=None), dict(codes=None), dict(scale=None), dict(rows=0), dict(rows=-1),
                    dict(cols=0), dict(cols=12), dict(ldw=63), dict(codes=264), dict(scale=257),
                    dict(W=258), dict(type=1, W=257), dict(rows=1 << 31, cols=64)):
            assert f(**bad) == EINVAL, bad
        for bad in (dict(group=0), dict(group=16), dict(group=96), dict(group=1024), dict(type=3),
                    dict(type=-1)):
            assert f(**bad) == EUNSUPPORTED, bad


def test_gemv_argument_errors(sq, L):
    def gemv(codes=256, scale=256, zero=None, rows=4, cols=64, group=32, nvec=1, x=256, xt=2, ldx=64,
             y=256, yt=2, ldy=4, ws=256, nws=1 << 30):
        return L.seedq_q4_gemv(codes, scale, zero, rows, cols, group, nvec, x, xt, ldx, y, yt, ldy,
                               ws, nws, None)

    for bad in (dict(x=None), dict(y=None), dict(codes=None), dict(scale=None), dict(nvec=-1),
                dict(cols=60), dict(rows=0), dict(ldx=63), dict(ldy=3), dict(x=257), dict(y=257),
                dict(xt=0, yt=0, x=258), dict(yt=0, y=258), dict(codes=8), dict(nvec=1 << 25)):
        assert gemv(**bad) == EINVAL, bad
    for bad in (dict(group=33), dict(xt=7), dict(yt=7), dict(xt=0, yt=1), dict(xt=1, yt=2)):
        assert gemv(**bad) == EUNSUPPORTED, bad
    assert gemv(nvec=0, x=None, y=None) == 0          # nothing to do
    for rows, cols, nvec, xt in ((4096, 4096, 64, 0), (4096, 4096, 512, 2)):
        need = sq.seedq_q4_gemv_workspace_bytes(rows, cols, nvec, xt)
        if need:
            a = dict(rows=rows, cols=cols, nvec=nvec, xt=xt, yt=0, ldx=cols, ldy=rows)
            assert gemv(**a, ws=None, nws=need) == EWORKSPACE
            assert gemv(**a, nws=need - 1) == EWORKSPACE
            assert gemv(**a, ws=264, nws=need) == EWORKSPACE
    assert sq.seedq_q4_gemv_workspace_bytes(0, 64, 1, 0) == 0
    assert sq.seedq_q4_gemv_workspace_bytes(4, 64, 0, 0) == 0


def test_logprobs_argument_errors(sq, L):
    def fwd(x=256, type=0, ld=100, rows=3, vocab=100, tok=256, top=2, lp=256, ent=256, lse=256,
            tt=256, tl=256, ws=256, nws=1 << 30):
        return L.seedq_token_logprobs(x, type, ld, rows, vocab, tok, top, lp, ent, lse, tt, tl, ws,
                                      nws, None)

    for bad in (dict(x=None), dict(ld=99), dict(rows=-1), dict(vocab=0), dict(tok=None),
                dict(top=-1), dict(top=33), dict(tt=None), dict(tl=None), dict(top=0),
                dict(lp=None, ent=None, lse=None, top=0, tt=None, tl=None), dict(x=258),
                dict(tok=260), dict(lp=258), dict(ent=258), dict(lse=258), dict(tt=260),
                dict(tl=258), dict(vocab=1 << 31, ld=1 << 31)):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(type=3) == EUNSUPPORTED
    assert fwd(rows=0, x=None, tok=None, lp=None, ent=None, lse=None, tt=None, tl=None) == 0
    need = sq.seedq_token_logprobs_workspace_bytes(1, 1 << 20, 5)
    if need:
        a = dict(rows=1, vocab=1 << 20, ld=1 << 20, top=5)
        assert fwd(**a, ws=None, nws=need) == EWORKSPACE
        assert fwd(**a, nws=need - 1) == EWORKSPACE
        assert fwd(**a, ws=264, nws=need) == EWORKSPACE

    def bwd(x=256, type=0, ld=100, rows=3, vocab=100, tok=256, lse=256, ent=256, g=256, h=256,
            out=512, ldg=100):
        return L.seedq_token_logprobs_backward(x, type, ld, rows, vocab, tok, lse, ent, g, h, out,
                                               ldg, None)

    for bad in (dict(x=None), dict(lse=None), dict(out=None), dict(g=None, h=None), dict(tok=None),
                dict(ent=None), dict(ld=99), dict(ldg=99), dict(out=256, ldg=101), dict(x=258),
                dict(out=514), dict(tok=260), dict(lse=258), dict(g=258), dict(h=258),
                dict(rows=-1), dict(vocab=0)):
        assert bwd(**bad) == EINVAL, bad
    assert bwd(type=4) == EUNSUPPORTED
    assert bwd(rows=0, x=None, lse=None, out=None) == 0


def test_helpers_refuse_what_is_not_theirs(sq):
    import torch
    W = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        sq.q4_quantize(W)                               # not on a GPU
    with pytest.raises(TypeError):
        sq.q4_quantize(W.double())
    with pytest.raises(ValueError):
        sq.q4_quantize(W[0])
    with pytest.raises(ValueError):
        sq.q4_quantize(W, group=48)
    q = sq.Q4Weights(torch.zeros(4, 8, dtype=torch.int32), torch.zeros(4, 1).half(), None, 4, 64, 128)
    with pytest.raises(ValueError):
        sq.q4_dequantize(q)
    with pytest.raises(TypeError):
        sq.q4_dequantize(q, torch.int32)
    with pytest.raises(ValueError):
        sq.q4_gemv(q, torch.zeros(3, 56))               # another number of columns
    with pytest.raises(ValueError):
        sq.q4_gemv(q, torch.zeros(3, 64))               # not on a GPU
    with pytest.raises(TypeError):
        sq.q4_gemv(q, torch.zeros(3, 64), torch.float16)
    x = torch.zeros(3, 10)
    with pytest.raises(ValueError):
        sq.token_logprobs(x, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError):
        sq.token_logprobs(x.int())
    with pytest.raises(ValueError):
        sq.token_logprobs(x[0])
    with pytest.raises(ValueError):
        sq.token_logprobs_backward(x, None, torch.zeros(3))


# ---------------------------------------------------------------- the oracle by hand

def test_oracle_quantiser_by_hand():
    w = np.zeros((1, 40))
    w[0, :4] = (7.0, -3.5, 0.5, 1.5)        # scale 1: ties to even
    w[0, 32:36] = (-1.0, 2.0, 0.0, 0.25)    # second, short group
    codes, scale, zero = oq4.quantize(w, 32, False)
    assert scale[0].tolist() == [1.0, float(np.float16(np.float32(2.0) / np.float32(7.0)))]
    assert codes[0, :5].tolist() == [15, 4, 8, 10, 8]
    codes, scale, zero = oq4.quantize(w, 32, True)
    assert scale[0, 0] == np.float16(10.5 / 15) and zero[0].tolist() == [5, 5]
    assert codes[0, 32:36].tolist() == [0, 15, 5, 6]
    assert np.array_equal(oq4.values(codes, scale, zero, 32)[0, 32:36],
                          (codes[0, 32:36] - 5.0) * float(scale[0, 1]))
    words = oq4.pack(codes)
    assert words.shape == (1, 8) and words[0, 4] == 0x5555_65F0 and not words[0, 5:].any()
    w[0, 5] = np.inf
    codes, scale, _ = oq4.quantize(w, 32, False)
    assert np.isnan(scale[0, 0]) and not codes[0, :32].any() and np.isfinite(scale[0, 1])


def test_oracle_logprobs_by_hand():
    lp, ent, lse, top = olp.row([0.0, 0.0, 0.0, 0.0], 2, 2)
    assert abs(lp + np.log(4)) < 1e-15 and abs(ent - np.log(4)) < 1e-15
    assert [t for t, _ in top] == [0, 1]
    inf = np.inf
    assert olp.row([-inf, -inf], 0, 1) == (-inf, 0.0, -inf, [(-1, -inf)])
    assert olp.row([-inf, 3.0], 0, 2) == (-inf, 0.0, 3.0, [(1, 0.0), (-1, -inf)])
    assert np.isnan(olp.row([inf, 3.0], 1, 1)[0]) and olp.row([inf, 3.0], -1, 1)[0] == 0.0
    # the gradient against differences of the value
    rng = np.random.default_rng(3)
    x = rng.normal(0, 2, 17)
    g, h, tok, d = 0.7, -0.3, 5, 1e-5
    _, ent, lse, _ = olp.row(x, tok, 0)
    grad = olp.gradient(x, tok, lse, ent, g, h)
    for v in range(17):
        e = np.zeros(17)
        e[v] = d
        a, b = olp.row(x + e, tok, 0), olp.row(x - e, tok, 0)
        diff = (g * (a[0] - b[0]) + h * (a[1] - b[1])) / (2 * d)
        assert abs(diff - grad[v]) < 1e-9
