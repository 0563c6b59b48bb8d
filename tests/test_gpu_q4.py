"""Weights in 4 bits with group scales on the GPU against the oracle.

Bars: codes, scales, zero points and words equal; decoded weights equal bit for bit
(the product has at most 15 significant bits, so fp32 holds it and a 16-bit result is
one rounding of it). Products: fp32 results of zero-mean vectors within 1e-6 of the
result in the 2-norm. A group of 128 adds terms whose running sum has an rms of at
most 100 |x| (codes 0 .. 15 without their zero point) against a result of 52 |x|,
each of some 8 roundings being 2^-24 / sqrt(12) of it: 1.3e-7, five times less than
the bar; sums over groups, random among themselves, keep the ratio and add
sqrt(groups) 2^-24 / sqrt(12), under 1e-7. 16-bit results may differ by their own half
unit (2^-8 and 2^-11 of the value) on top of that. For single elements the bar is
12 standard deviations of the same error."""
import numpy as np
import pytest

from oracle import q4 as oq4

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")
UNIT = {"float32": 0.0, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


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


def _random_q4(sq, torch, rng, rows, cols, group, zeros):
    """Random codes with scales of one magnitude, and their exact values."""
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    G = -(-cols // group)
    scale = rng.uniform(0.002, 0.006, (rows, G)).astype(np.float16)
    zero = rng.integers(0, 16, (rows, G)).astype(np.uint8) if zeros else None
    words = torch.from_numpy(oq4.pack(codes).view(np.int32)).cuda()
    q = sq.Q4Weights(words, torch.from_numpy(scale).cuda(),
                     None if zero is None else torch.from_numpy(zero).cuda(), rows, cols, group)
    return q, oq4.values(codes, scale, zero, group)


def _check_product(y, exact, dtype):
    y = y.double().cpu().numpy()
    assert y.shape == exact.shape
    err = np.abs(y - exact)
    norm = np.linalg.norm(exact)
    bar = 1e-6 * norm + UNIT[dtype] * norm
    assert np.linalg.norm(err) <= bar, np.linalg.norm(err) / max(norm, 1e-300)
    rms = norm / np.sqrt(exact.size)
    assert np.all(err <= 12e-6 * rms + UNIT[dtype] * np.abs(exact) * 1.001)


# ---------------------------------------------------------------- quantiser and decoder

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,cols,group", [(1, 8, 32), (3, 40, 32), (5, 136, 64), (7, 520, 128),
                                             (4, 1032, 256), (2, 2056, 512), (9, 512, 512)])
def test_quantise_matches_the_definition(sq, torch, rows, cols, group, zeros, dtype):
    rng = np.random.default_rng(rows * cols + group)
    w = (rng.normal(0, 0.02, (rows, cols)) * np.exp(rng.normal(0, 2, (rows, 1)))).astype(np.float32)
    w[0, : min(cols, 16)] = 0.0
    if rows > 2:
        w[1] = 0.0                                   # scale 0
        w[2, :8] = np.linspace(-7, 7, 8) / 2         # ties where the largest is 3.5
        w[2, 8:group] = 0.0
    if rows > 3:
        w[3] = np.abs(w[3]) + 1.0                    # one sign: the zero point is at the end
    if rows > 4:
        w[4] *= 2e-7                                 # scales among fp16's subnormals
    t = torch.from_numpy(w).to(getattr(torch, dtype))
    q = sq.q4_quantize(t.cuda(), group, zeros=zeros)
    codes, scale, zero = oq4.quantize(t.double().numpy(), group, zeros)
    assert np.array_equal(q.scale.cpu().numpy().view(np.uint16), scale.view(np.uint16))
    assert np.array_equal(q.codes.cpu().numpy().view(np.uint32), oq4.pack(codes))
    assert (q.zero is None) == (zero is None)
    if zeros:
        assert np.array_equal(q.zero.cpu().numpy(), zero)
    back = sq.q4_dequantize(q).cpu().numpy()
    assert np.array_equal(back, oq4.values(codes, scale, zero, group).astype(np.float32))


def test_quantise_near_ties_and_extremes(sq, torch):
    # quotients next to every tie, at the fp32 neighbours of the tie: the code is the
    # rounding of the fp32 quotient
    rng = np.random.default_rng(5)
    rows = 64
    w = np.zeros((rows, 32), np.float32)
    top = rng.uniform(0.01, 3, rows).astype(np.float32)
    s = (top / np.float32(7)).astype(np.float16).astype(np.float32)
    for r in range(rows):
        ties = (np.arange(-7, 8) + 0.5).astype(np.float32) * s[r]
        w[r, 0] = top[r]
        near = np.concatenate([np.nextafter(ties, -np.float32(9)), np.nextafter(ties, np.float32(9))])
        near = near[np.abs(near) <= top[r]]
        w[r, 1:1 + near.size] = near[:31]
    q = sq.q4_quantize(torch.from_numpy(w).cuda(), 32)
    codes, scale, _ = oq4.quantize(w, 32, False)
    assert np.array_equal(q.codes.cpu().numpy().view(np.uint32), oq4.pack(codes))
    # the scale is capped, groups that are not finite decode to NaN and leave the others alone
    w = np.ones((4, 64), np.float32)
    w[0, 3], w[1, 40], w[2, 5], w[3, 7] = 3e38, np.inf, np.nan, -3e38
    w[0, 4] = -3e38
    for zeros in (False, True):
        q = sq.q4_quantize(torch.from_numpy(w).cuda(), 32, zeros=zeros)
        codes, scale, zero = oq4.quantize(w, 32, zeros)
        assert np.array_equal(q.codes.cpu().numpy().view(np.uint32), oq4.pack(codes))
        got = q.scale.cpu().numpy()
        assert np.array_equal(got, scale, equal_nan=True) and got[0, 0] == 65504.0
        back = sq.q4_dequantize(q).cpu().numpy()
        assert np.isnan(back[1, 32:]).all() and np.isnan(back[2, :32]).all()
        assert np.isfinite(back[1, :32]).all() and np.isfinite(back[2, 32:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,cols,group", [(1, 8, 32), (3, 72, 32), (17, 1032, 128), (6, 4096, 512),
                                             (1001, 264, 64)])
def test_dequantise_is_exact(sq, torch, rows, cols, group, zeros, dtype):
    q, W = _random_q4(sq, torch, np.random.default_rng(cols), rows, cols, group, zeros)
    dt = getattr(torch, dtype)
    got = sq.q4_dequantize(q, dt)
    ref = torch.from_numpy(W).float().to(dt)
    assert got.dtype == dt and torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_and_dequantise_of_rows_anywhere(sq, torch, dtype):
    # a view with another row stride and an odd first element; outputs inside a larger
    # buffer whose other elements stay
    dt = getattr(torch, dtype)
    rows, cols, group = 5, 200, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.randn(rows, cols + 13, device="cuda", generator=g).to(dt)
    view = big[:, 3:3 + cols]
    q, p = sq.q4_quantize(view, group), sq.q4_quantize(view.contiguous(), group)
    assert torch.equal(q.codes, p.codes) and torch.equal(q.scale, p.scale)
    turned = sq.q4_quantize(view.contiguous().t().contiguous().t(), group)
    assert torch.equal(turned.codes, p.codes)
    out = torch.full((rows, cols + 13), 7.0, dtype=dt, device="cuda")
    code = {"float32": 0, "float16": 1, "bfloat16": 2}[dtype]
    sq.seedq_q4_dequantize(q.codes, q.scale, None, rows, cols, group, out[:, 3:], code, cols + 13)
    assert torch.equal(out[:, 3:3 + cols], sq.q4_dequantize(q, dt))
    assert (out[:, :3] == 7.0).all() and (out[:, 3 + cols:] == 7.0).all()


# ---------------------------------------------------------------- products

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, False), (128, True), (256, True),
                                         (512, False)])
@pytest.mark.parametrize("rows,cols,nvec", [(1, 8, 1), (5, 40, 3), (33, 264, 1), (16, 128, 16),
                                            (100, 1032, 2), (257, 2056, 5), (130, 648, 17),
                                            (64, 4096, 33)])
def test_product_matches_64_bits(sq, torch, rows, cols, nvec, group, zeros, dtype):
    rng = np.random.default_rng(rows + cols + nvec)
    q, W = _random_q4(sq, torch, rng, rows, cols, group, zeros)
    dt = getattr(torch, dtype)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(dt)
    exact = x.double().numpy() @ W.T
    for out in {dt, torch.float32}:
        y = sq.q4_gemv(q, x.cuda(), out)
        assert y.dtype == out and y.shape == (nvec, rows)
        _check_product(y, exact, str(out).split(".")[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,nvec,group,zeros",
                         [(300, 1096, 64, 128, True), (129, 2056, 65, 64, False),
                          (384, 520, 130, 32, True), (1000, 4096, 257, 128, False),
                          (64, 136, 1000, 128, True), (2049, 264, 96, 256, False)])
def test_product_of_many_vectors(sq, torch, rows, cols, nvec, group, zeros, dtype):
    rng = np.random.default_rng(rows + cols + nvec)
    q, W = _random_q4(sq, torch, rng, rows, cols, group, zeros)
    dt = getattr(torch, dtype)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(dt)
    exact = x.double().numpy() @ W.T
    for out in {dt, torch.float32}:
        _check_product(sq.q4_gemv(q, x.cuda(), out), exact, str(out).split(".")[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_long_and_wide_matrices(sq, torch, dtype):
    # a long row for few rows, and many rows of one word
    rng = np.random.default_rng(9)
    dt = getattr(torch, dtype)
    for rows, cols, nvec in ((3, 65544, 1), (2, 32768, 9), (70001, 8, 2), (20000, 32, 40)):
        q, W = _random_q4(sq, torch, rng, rows, cols, 128, True)
        x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(dt)
        _check_product(sq.q4_gemv(q, x.cuda(), torch.float32), x.double().numpy() @ W.T, "float32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 3, 8, 40, 200])
def test_product_with_vectors_anywhere(sq, torch, nvec, dtype):
    # x in rows of an odd stride from an odd element; y inside a larger buffer; the
    # results equal those of dense buffers, and nothing else is written
    rng = np.random.default_rng(nvec)
    rows, cols, group = 77, 328, 64
    q, _ = _random_q4(sq, torch, rng, rows, cols, group, True)
    dt = getattr(torch, dtype)
    big = torch.from_numpy(rng.normal(0, 1, (nvec, cols + 9)).astype(np.float32)).to(dt).cuda()
    big[:, :5] = float("nan")                        # never read
    big[:, 5 + cols:] = float("nan")
    view = big[:, 5:5 + cols]
    ref = sq.q4_gemv(q, view.contiguous())
    assert torch.equal(sq.q4_gemv(q, view), ref)
    assert torch.equal(sq.q4_gemv(q, view.contiguous().t().contiguous().t()), ref)
    code = {"float32": 0, "float16": 1, "bfloat16": 2}[dtype]
    out = torch.full((nvec, rows + 3), 7.0, dtype=dt, device="cuda")
    nws = sq.seedq_q4_gemv_workspace_bytes(rows, cols, nvec, code)
    ws = torch.empty(max(nws, 256), dtype=torch.uint8, device="cuda")
    sq.seedq_q4_gemv(q.codes, q.scale, q.zero, rows, cols, group, nvec, view, code,
                     view.stride(0), out[:, 1:], code, rows + 3, ws, nws)
    assert torch.equal(out[:, 1:1 + rows], ref)
    assert (out[:, 0] == 7.0).all() and (out[:, 1 + rows:] == 7.0).all()
    if nvec == 1:
        assert torch.equal(sq.q4_gemv(q, view[0]), ref[0])
    assert sq.q4_gemv(q, view[:0]).shape == (0, rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 4, 24, 160])
def test_products_are_a_function_of_the_inputs(sq, torch, nvec, dtype):
    # the same bits from run to run, on another stream, and with other memory in the
    # workspace
    rng = np.random.default_rng(nvec)
    q, _ = _random_q4(sq, torch, rng, 513, 1544, 128, True)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, 1544)).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    ref = sq.q4_gemv(q, x)
    torch.cuda.synchronize()
    junk = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    del junk
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = sq.q4_gemv(q, x, stream=s)
    s.synchronize()
    assert torch.equal(other, ref)
    for _ in range(3):
        assert torch.equal(sq.q4_gemv(q, x), ref)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 6, 48, 144])
def test_vectors_that_are_not_finite_stay_apart(sq, torch, nvec, dtype):
    # one vector with an infinity or a NaN does not touch the others; a NaN scale makes
    # its row NaN and no other
    rng = np.random.default_rng(nvec)
    rows, cols = 40, 520
    q, W = _random_q4(sq, torch, rng, rows, cols, 128, False)
    q.codes[:] &= 0x77777777                        # u < 8: no value is zero
    W = sq.q4_dequantize(q).double().cpu().numpy()
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(getattr(torch, dtype))
    exact = x.double().numpy() @ W.T
    bad = x.clone()
    bad[nvec // 2, 100] = float("inf")
    y = sq.q4_gemv(q, bad.cuda(), torch.float32).cpu().double().numpy()
    keep = np.arange(nvec) != nvec // 2
    assert not np.isfinite(y[~keep]).any()
    if keep.any():
        _check_product(torch.from_numpy(y[keep]), exact[keep], "float32")
    q.scale[7, 2] = float("nan")
    y = sq.q4_gemv(q, x.cuda(), torch.float32).cpu().double().numpy()
    rest = np.arange(rows) != 7
    assert np.isnan(y[:, 7]).all()
    _check_product(torch.from_numpy(y[:, rest]), exact[:, rest], "float32")


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("nvec", [1, 5, 40, 150])
def test_small_and_large_magnitudes(sq, torch, nvec, dtype):
    # whole vectors scaled by a power of two: the results scale exactly with them
    rng = np.random.default_rng(nvec)
    q, W = _random_q4(sq, torch, rng, 50, 264, 64, True)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, 264)).astype(np.float32)).to(getattr(torch, dtype))
    for e in ((-6, 6) if dtype == "float16" else (-40, 40)):
        xs = (x.float() * 2.0 ** e).to(x.dtype)
        _check_product(sq.q4_gemv(q, xs.cuda(), torch.float32), xs.double().numpy() @ W.T, "float32")


@pytest.mark.parametrize("nvec,dtype", [(1, "bfloat16"), (2, "float32"), (9, "float16"),
                                        (200, "bfloat16"), (100, "float32")])
def test_products_in_a_graph(sq, torch, nvec, dtype):
    # a captured call replayed on new inputs, with other work between the replays
    rng = np.random.default_rng(nvec)
    q, _ = _random_q4(sq, torch, rng, 300, 1032, 128, True)
    dt = getattr(torch, dtype)
    xs = [torch.from_numpy(rng.normal(0, 1, (nvec, 1032)).astype(np.float32)).to(dt).cuda()
          for _ in range(4)]
    x = xs[0].clone()
    refs = [sq.q4_gemv(q, v).clone() for v in xs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sq.q4_gemv(q, x)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sq.q4_gemv(q, x)
    for v, ref in zip(xs, refs):
        x.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref)
        torch.randn(1 << 20, device="cuda").sum().item()


def test_offsets_past_32_bits(sq, torch):
    # 2^31 weights in 2^30 bytes of codes: the last rows' codes, scales, decoded weights
    # (8 GiB in fp32) and products
    rows, cols, group = (1 << 17) + 8, 1 << 14, 128
    codes = torch.zeros((rows, cols // 8), dtype=torch.int32, device="cuda")
    codes[-1] = 0x77777777                           # value -1 times the scale
    codes[:-1] = -2004318072                         # 0x88888888: zero
    scale = torch.full((rows, cols // group), 0.5, dtype=torch.float16, device="cuda")
    q = sq.Q4Weights(codes, scale, None, rows, cols, group)
    x = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda")
    for nvec in (1, 20, 130):
        y = sq.q4_gemv(q, x.expand(nvec, cols).contiguous(), torch.float32)
        assert (y[:, -1] == -0.5 * cols).all() and (y[:, :-1] == 0).all()
    W = sq.q4_dequantize(q, torch.float32)
    assert (W[-1] == -0.5).all() and not W[-2].any() and not W[rows // 2].any()
    p = sq.q4_quantize(W, group)
    assert torch.equal(sq.q4_dequantize(p, torch.bfloat16)[-3:].float(), W[-3:])


def test_helpers_refuse_wrong_tensors(sq, torch):
    q, _ = _random_q4(sq, torch, np.random.default_rng(0), 8, 64, 32, True)
    x = torch.zeros(2, 64, device="cuda")
    bad = [sq.Q4Weights(q.codes[:4], q.scale, q.zero, 8, 64, 32),
           sq.Q4Weights(q.codes, q.scale[:, :1], q.zero, 8, 64, 32),
           sq.Q4Weights(q.codes, q.scale.float(), q.zero, 8, 64, 32),
           sq.Q4Weights(q.codes, q.scale, q.zero.int(), 8, 64, 32),
           sq.Q4Weights(q.codes, q.scale.cpu(), q.zero, 8, 64, 32),
           sq.Q4Weights(q.codes.t().contiguous().t(), q.scale, q.zero, 8, 64, 32)]
    for b in bad:
        with pytest.raises(ValueError):
            sq.q4_gemv(b, x)
        with pytest.raises(ValueError):
            sq.q4_dequantize(b)
    with pytest.raises(ValueError):
        sq.q4_gemv(q, x.cpu())
    with pytest.raises(sq.SeedqError) as e:
        sq.q4_gemv(sq.Q4Weights(q.codes, q.scale, q.zero, 8, 64, 48), x)
    assert e.value.code == -2
    with pytest.raises(sq.SeedqError) as e:
        sq.q4_quantize(torch.zeros(4, 12, device="cuda"))
    assert e.value.code == -1
