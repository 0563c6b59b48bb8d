"""Matrices of microscaled 4-bit floats on the GPU against the oracle.

Bars: codes, exponents and words equal; decoded weights equal bit for bit. Products: the
terms are exact, so an output errs by the roundings of its partial sums alone. A partial sum
takes part in at most D = 48 + ncols / 8 of them one after another (a lane's 32 columns, a
tree over lanes and waves, the steps of at least 16 columns of a matrix product with two
roundings each, the joins), and each is at most 2^-24 of a number below mag = sum |w x|: no
output errs by more than D 2^-24 mag. Of vectors of both signs the partial sums have an rms of
at most q = sqrt(sum (w x)^2) and a rounding one of 2^-24 / sqrt(3) of its sum, so the errors
of all outputs have the 2-norm of sqrt(D / 3) 2^-24 q; the bar is (4 + sqrt(D)) 2^-24 q, the
4 for products with few outputs. Outputs in 16 bits differ by their own half unit (2^-8 and
2^-11 of the value, 2^-25 among fp16's subnormals) on top of that."""
import numpy as np
import pytest

from oracle import mx4 as omx
from oracle import q4 as oq4
from test_gpu_q4 import TYPES, UNIT, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def random_mx4(sq, torch, rng, rows, cols, lo=118, hi=124):  # noqa: F811
    """Random codes with exponents lo .. hi, and their exact values."""
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    scale = rng.integers(lo, hi + 1, (rows, -(-cols // 32))).astype(np.uint8)
    words = torch.from_numpy(oq4.pack(codes).view(np.int32)).cuda()
    return sq.Mx4Weights(words, torch.from_numpy(scale).cuda(), rows, cols), omx.values(codes, scale)


def check_product(y, x, W, dtype, both_signs=True):
    y = y.double().cpu().numpy()
    exact, mag = x @ W.T, np.abs(x) @ np.abs(W).T
    assert y.shape == exact.shape
    D = 48 + x.shape[1] / 8
    own = UNIT[dtype] * np.abs(exact) * 1.001 + (2.0 ** -25 if dtype == "float16" else 0.0)
    err = np.maximum(np.abs(y - exact) - own, 0.0)
    assert np.all(err <= D * 2.0 ** -24 * mag), np.max(err / np.maximum(mag, 1e-300)) * 2.0 ** 24
    if both_signs:
        q = np.sqrt((x * x) @ (W * W).T)
        assert np.linalg.norm(err) <= (4 + np.sqrt(D)) * 2.0 ** -24 * np.linalg.norm(q)


# ---------------------------------------------------------------- quantiser and decoder

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 40), (5, 136), (7, 520), (4, 1032), (2, 2056)])
def test_quantise_matches_the_definition(sq, torch, rows, cols, dtype):  # noqa: F811
    rng = np.random.default_rng(rows * cols)
    w = (rng.normal(0, 0.02, (rows, cols)) * np.exp(rng.normal(0, 2, (rows, 1)))).astype(np.float32)
    w[0, :min(cols, 16)] = 0.0
    w[0, 1] = -0.0
    if rows > 2:
        w[1] = 0.0
        # every tie, its neighbours, and what saturates, under exponents 0 and 4
        t = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6.5, 7, 7.9375], np.float32)
        t = np.concatenate([t, -t, [4.0]])
        w[2, :21] = t
        w[2, 21:32] = 0.0
        if cols > 40:
            near = np.concatenate([np.nextafter(t[:7], np.float32(0)), np.nextafter(t[:7], np.float32(9)),
                                   t[:7], [7.0]]).astype(np.float32)
            w[2, 32:54] = 16 * near
            w[2, 54:64] = 0.0
    if rows > 3:
        w[3] *= np.float32(2.0 ** -12)                # among fp16's subnormals
    if rows > 4 and dtype != "float16":
        w[4] *= np.float32(2.0 ** -118)               # among fp32's subnormals
    t = torch.from_numpy(w).to(getattr(torch, dtype))
    q = sq.mx4_quantize(t.cuda())
    codes, scale = omx.quantize(t.double().numpy())
    assert np.array_equal(q.scale.cpu().numpy(), scale)
    assert np.array_equal(q.codes.cpu().numpy().view(np.uint32), oq4.pack(codes))
    back = sq.mx4_dequantize(q).cpu().numpy()
    ref = omx.values(codes, scale).astype(np.float32)
    assert np.array_equal(back, ref) and np.array_equal(np.signbit(back), np.signbit(ref))


def test_quantise_the_whole_range_and_what_is_not_finite(sq, torch):  # noqa: F811
    w = np.ones((6, 64), np.float32)
    w[0, 3], w[1, 40], w[2, 5], w[3, 7] = 3.4e38, np.inf, np.nan, -3e38
    w[4] = 1e-45
    w[5, :32] = 2.0 ** -126
    w[5, 32:] = np.float32(2.0 ** -127) * np.arange(32)
    q = sq.mx4_quantize(torch.from_numpy(w).cuda())
    codes, scale = omx.quantize(w)
    assert np.array_equal(q.scale.cpu().numpy(), scale) and scale[0, 0] == 252
    assert np.array_equal(q.codes.cpu().numpy().view(np.uint32), oq4.pack(codes))
    back = sq.mx4_dequantize(q).cpu().numpy()
    assert np.isnan(back[1, 32:]).all() and np.isnan(back[2, :32]).all()
    assert np.isfinite(back[1, :32]).all() and np.isfinite(back[2, 32:]).all()
    assert np.array_equal(back, omx.values(codes, scale).astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,lo,hi", [(1, 8, 118, 124), (3, 72, 90, 150), (17, 1032, 0, 252),
                                             (1001, 264, 110, 140)])
def test_dequantise_is_exact(sq, torch, rows, cols, lo, hi, dtype):  # noqa: F811
    q, W = random_mx4(sq, torch, np.random.default_rng(cols), rows, cols, lo, hi)
    dt = getattr(torch, dtype)
    got = sq.mx4_dequantize(q, dt)
    ref = torch.from_numpy(W).float().to(dt)
    assert got.dtype == dt and torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_and_dequantise_of_rows_anywhere(sq, torch, dtype):  # noqa: F811
    dt = getattr(torch, dtype)
    rows, cols = 5, 200
    base = torch.randn(rows * 211 + 7, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    view = base[3:3 + rows * 211].view(rows, 211)[:, 1:1 + cols]
    q = sq.mx4_quantize(view)
    ref = sq.mx4_quantize(view.contiguous())
    assert torch.equal(q.codes, ref.codes) and torch.equal(q.scale, ref.scale)
    code = {"float32": 0, "float16": 1, "bfloat16": 2}[dtype]
    buf = torch.full((rows * 211 + 7,), 9.0, dtype=dt, device="cuda")
    sq.seedq_mx4_dequantize(q.codes, q.scale, rows, cols, buf[5:], code, 211)
    out = buf[5:5 + rows * 211].view(rows, 211)
    assert torch.equal(out[:, :cols], sq.mx4_dequantize(q, dt))
    assert (out[:, cols:] == 9).all() and (buf[:5] == 9).all() and (buf[5 + rows * 211:] == 9).all()


# ---------------------------------------------------------------- products with vectors

SHAPES = [(1, 8), (3, 40), (33, 520), (100, 2056), (1001, 264), (257, 4096)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 2, 3, 4, 5, 8, 11, 16, 17, 33, 100])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gemv(sq, torch, rows, cols, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(rows + cols + nvec)
    q, W = random_mx4(sq, torch, rng, rows, cols)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols))).to(getattr(torch, dtype))
    for out in {dtype, "float32"}:
        y = sq.mx4_gemv(q, x.cuda(), getattr(torch, out))
        assert y.dtype == getattr(torch, out)
        check_product(y, x.double().numpy(), W, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,nvec", [(9000, 520, 5), (9000, 520, 40), (70, 20480, 1), (70, 20480, 9),
                                            (70, 20480, 40), (4100, 1032, 300), (16400, 264, 2),
                                            (520, 66000, 2)])
def test_gemv_of_other_cuts(sq, torch, rows, cols, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(rows)
    q, W = random_mx4(sq, torch, rng, rows, cols)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols))).to(getattr(torch, dtype))
    y = sq.mx4_gemv(q, x.cuda(), torch.float32)
    check_product(y, x.double().numpy(), W, "float32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 6, 40])
def test_gemv_of_one_sign(sq, torch, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(nvec)
    q, W = random_mx4(sq, torch, rng, 70, 4096)
    x = torch.from_numpy(rng.uniform(0.5, 1, (nvec, 4096))).to(getattr(torch, dtype))
    q.codes &= 0x77777777
    y = sq.mx4_gemv(q, x.cuda(), torch.float32)
    check_product(y, x.double().numpy(), np.abs(W), "float32", both_signs=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 6, 40])
def test_gemv_of_far_exponents(sq, torch, nvec, dtype):  # noqa: F811
    # blocks 2^-60 .. 2^60 of each other, and vectors that make the small ones count
    rng = np.random.default_rng(nvec)
    rows, cols = 40, 520
    q, W = random_mx4(sq, torch, rng, rows, cols, 67, 187)
    x = rng.normal(0, 1, (nvec, cols))
    x[:, 32:] = 0.0
    if dtype == "float16":
        x[:, 32:64] = rng.normal(0, 1000, (nvec, 32))
    x = torch.from_numpy(x).to(getattr(torch, dtype))
    y = sq.mx4_gemv(q, x.cuda(), torch.float32)
    check_product(y, x.double().numpy(), W, "float32")
    # the ends of the range, where fp32 holds the products
    small = random_mx4(sq, torch, rng, rows, cols, 0, 3)
    x = torch.full((nvec, cols), 8.0, dtype=getattr(torch, dtype))
    assert torch.equal(sq.mx4_gemv(small[0], x.cuda(), torch.float32).cpu(),
                       torch.from_numpy(x.double().numpy() @ small[1].T).float())
    large = random_mx4(sq, torch, rng, rows, 32, 250, 252)
    x = torch.zeros((nvec, 32), dtype=getattr(torch, dtype))
    x[:, 5] = 2.0 ** -10
    assert torch.equal(sq.mx4_gemv(large[0], x.cuda(), torch.float32).cpu(),
                       torch.from_numpy(x.double().numpy() @ large[1].T).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 6, 40])
def test_gemv_what_is_not_finite_stays_in_its_row(sq, torch, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(3)
    q, W = random_mx4(sq, torch, rng, 70, 264)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, 264))).to(getattr(torch, dtype)).cuda()
    clean = sq.mx4_gemv(q, x)
    q.scale[5, 3] = 255
    y = sq.mx4_gemv(q, x)
    assert torch.isnan(y[:, 5]).all()
    y[:, 5] = clean[:, 5]
    assert torch.equal(y, clean)
    q.scale[5, 3] = 120
    clean = sq.mx4_gemv(q, x)
    for bad in (float("nan"), float("inf")):
        z = x.clone()
        z[nvec // 2, 100] = bad
        y = sq.mx4_gemv(q, z)
        hit = W[:, 100] != 0
        assert not torch.isfinite(y[nvec // 2].cpu()[torch.from_numpy(hit)]).any()
        y[nvec // 2] = clean[nvec // 2]
        assert torch.equal(y, clean)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 2, 5, 20, 70])
def test_gemv_of_rows_anywhere(sq, torch, nvec, dtype):  # noqa: F811
    dt = getattr(torch, dtype)
    code = {"float32": 0, "float16": 1, "bfloat16": 2}[dtype]
    rng = np.random.default_rng(nvec)
    rows, cols = 131, 328
    q, W = random_mx4(sq, torch, rng, rows, cols)
    base = torch.from_numpy(rng.normal(0, 1, nvec * 349 + 9)).to(dt).cuda()
    x = base[3:3 + nvec * 349].view(nvec, 349)[:, :cols]
    ref = sq.mx4_gemv(q, x.contiguous())
    assert torch.equal(sq.mx4_gemv(q, x), ref)
    assert torch.equal(sq.mx4_gemv(q, x.flip(1).contiguous().flip(1)), ref)
    buf = torch.full((nvec * 150 + 7,), 9.0, dtype=dt, device="cuda")
    nws = sq.seedq_mx4_gemv_workspace_bytes(rows, cols, nvec, code)
    ws = torch.empty(nws + 256, dtype=torch.uint8, device="cuda") if nws else None
    sq.seedq_mx4_gemv(q.codes, q.scale, rows, cols, nvec, x, code, 349, buf[5:], code, 150, ws, nws)
    out = buf[5:5 + nvec * 150].view(nvec, 150)
    assert torch.equal(out[:, :rows], ref) and (out[:, rows:] == 9).all()
    assert (buf[:5] == 9).all() and (buf[5 + nvec * 150:] == 9).all()
    assert sq.mx4_gemv(q, base[:0].view(0, cols)).shape == (0, rows)
    assert torch.equal(sq.mx4_gemv(q, x[0]), sq.mx4_gemv(q, x[:1])[0])


# ---------------------------------------------------------------- products of two coded matrices

@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("na", [1, 2, 5, 16, 17, 33, 64, 100, 130])
@pytest.mark.parametrize("nb,cols", SHAPES + [(300, 72), (130, 8), (70, 12312)])
def test_matmul(sq, torch, na, nb, cols, out):  # noqa: F811
    rng = np.random.default_rng(na + nb + cols)
    a, A = random_mx4(sq, torch, rng, na, cols, 124, 129)
    b, B = random_mx4(sq, torch, rng, nb, cols, 114, 122)
    check_product(sq.mx4_matmul(a, b, getattr(torch, out)), A, B, out)


@pytest.mark.parametrize("na,nb,cols", [(700, 1100, 520), (1030, 260, 264), (300, 5000, 1032), (260, 300, 8200),
                                        (20, 4100, 4096), (3, 17000, 72)])
def test_matmul_of_other_cuts(sq, torch, na, nb, cols):  # noqa: F811
    rng = np.random.default_rng(na + nb)
    a, A = random_mx4(sq, torch, rng, na, cols, 124, 129)
    b, B = random_mx4(sq, torch, rng, nb, cols, 114, 122)
    check_product(sq.mx4_matmul(a, b), A, B, "float32")


def test_matmul_places_every_code(sq, torch):  # noqa: F811
    # one code in a row of a, one in a row of b: rows, columns and exponents show
    na, nb, cols = 40, 70, 200
    rng = np.random.default_rng(9)
    ca, cb = np.zeros((na, cols), np.uint8), rng.integers(0, 16, (nb, cols)).astype(np.uint8)
    ca[np.arange(na), rng.integers(0, cols, na)] = rng.integers(1, 8, na)
    sa = rng.integers(100, 150, (na, 7)).astype(np.uint8)
    sb = rng.integers(100, 150, (nb, 7)).astype(np.uint8)
    make = lambda c, s, n: sq.Mx4Weights(torch.from_numpy(oq4.pack(c).view(np.int32)).cuda(),  # noqa: E731
                                         torch.from_numpy(s).cuda(), n, cols)
    y = sq.mx4_matmul(make(ca, sa, na), make(cb, sb, nb))
    assert torch.equal(y.cpu(), torch.from_numpy(omx.values(ca, sa) @ omx.values(cb, sb).T).float())


def test_matmul_what_is_not_finite_and_the_ends_of_the_range(sq, torch):  # noqa: F811
    rng = np.random.default_rng(4)
    a, A = random_mx4(sq, torch, rng, 50, 520)
    b, B = random_mx4(sq, torch, rng, 90, 520)
    clean = sq.mx4_matmul(a, b)
    a.scale[7, 16] = 255
    b.scale[80, 0] = 255
    y = sq.mx4_matmul(a, b)
    assert torch.isnan(y[7]).all() and torch.isnan(y[:, 80]).all()
    y[7], y[:, 80] = clean[7], clean[:, 80]
    assert torch.equal(y, clean)
    a, A = random_mx4(sq, torch, rng, 50, 32, 0, 0)
    b, B = random_mx4(sq, torch, rng, 90, 32, 252, 252)
    assert torch.equal(sq.mx4_matmul(a, b).cpu(), torch.from_numpy(A @ B.T).float())


def test_matmul_into_a_larger_buffer(sq, torch):  # noqa: F811
    rng = np.random.default_rng(6)
    for na, nb, cols, code in ((5, 70, 264, 0), (140, 300, 264, 2), (70, 33, 40, 1)):
        a, _ = random_mx4(sq, torch, rng, na, cols)
        b, _ = random_mx4(sq, torch, rng, nb, cols)
        dt = (torch.float32, torch.float16, torch.bfloat16)[code]
        ref = sq.mx4_matmul(a, b, dt)
        ld = nb + 13
        buf = torch.full((na * ld + 8,), 9.0, dtype=dt, device="cuda")
        nws = sq.seedq_mx4_matmul_workspace_bytes(na, nb, cols)
        ws = torch.empty(nws, dtype=torch.uint8, device="cuda") if nws else None
        sq.seedq_mx4_matmul(a.codes, a.scale, na, b.codes, b.scale, nb, cols, buf[3:], code, ld, ws, nws)
        out = buf[3:3 + na * ld].view(na, ld)
        assert torch.equal(out[:, :nb], ref) and (out[:, nb:] == 9).all()
        assert (buf[:3] == 9).all() and (buf[3 + na * ld:] == 9).all()


# ---------------------------------------------------------------- streams, graphs, repeats

def test_on_another_stream_and_again(sq, torch):  # noqa: F811
    rng = np.random.default_rng(8)
    q, _ = random_mx4(sq, torch, rng, 600, 1032)
    W = torch.from_numpy(rng.normal(0, 1, (300, 1032))).float().cuda()
    side = torch.cuda.Stream()
    for nvec in (1, 9, 60):
        x = W[:nvec].bfloat16()
        torch.cuda.synchronize()
        ref = [sq.mx4_gemv(q, x), sq.mx4_matmul(sq.mx4_quantize(x), q)]
        torch.cuda.synchronize()
        got = [sq.mx4_gemv(q, x, stream=side), sq.mx4_matmul(sq.mx4_quantize(x, stream=side), q, stream=side)]
        side.synchronize()
        for a, b in zip(ref, got):
            assert torch.equal(a, b)
        for _ in range(3):
            assert torch.equal(sq.mx4_gemv(q, x), ref[0])


def test_in_a_graph(sq, torch):  # noqa: F811
    rng = np.random.default_rng(10)
    q, _ = random_mx4(sq, torch, rng, 600, 4096)
    xs = [torch.from_numpy(rng.normal(0, 1, (n, 4096))).bfloat16().cuda() for n in (1, 9, 60)]

    def step():
        return [t for x in xs for t in (sq.mx4_gemv(q, x), sq.mx4_matmul(sq.mx4_quantize(x), q))]

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for seed in range(3):
        for x in xs:
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


def test_helpers_refuse(sq, torch):  # noqa: F811
    q, _ = random_mx4(sq, torch, np.random.default_rng(1), 9, 72)
    x = torch.zeros(2, 72, device="cuda")
    for bad in (lambda: sq.mx4_gemv(q, x[:, :64]), lambda: sq.mx4_gemv(q, x.cpu()),
                lambda: sq.mx4_gemv(sq.Mx4Weights(q.codes[:, :8], q.scale, 9, 72), x),
                lambda: sq.mx4_gemv(sq.Mx4Weights(q.codes, q.scale[:8], 9, 72), x),
                lambda: sq.mx4_gemv(sq.Mx4Weights(q.codes, q.scale.int(), 9, 72), x),
                lambda: sq.mx4_gemv(sq.Mx4Weights(q.codes, q.scale, 9, 104), torch.zeros(2, 104, device="cuda")),
                lambda: sq.mx4_matmul(q, sq.Mx4Weights(q.codes[:, :8], q.scale[:, :2], 9, 64)),
                lambda: sq.mx4_dequantize(sq.Mx4Weights(q.codes.cpu(), q.scale, 9, 72))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sq.SeedqError):
        sq.mx4_quantize(torch.zeros(3, 12, device="cuda"))          # columns not in eights
    with pytest.raises(sq.SeedqError):                              # codes that are not at 16 bytes
        flat = torch.zeros(9 * 12 + 1, dtype=torch.int32, device="cuda")
        sq.mx4_gemv(sq.Mx4Weights(flat[1:].view(9, 12), q.scale, 9, 72), x)
    with pytest.raises(TypeError):
        sq.mx4_gemv(q, x.double())
