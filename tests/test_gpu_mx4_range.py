"""Products of matrices of microscaled 4-bit floats past the sizes of one launch, and vectors
at both ends of fp32's range.

Bars: where weights are multiples of 1/2 and vectors small whole numbers every sum is exact
in fp32, so results are equal. For the ends of the range, those of test_gpu_mx4, and 2^-133
of each weight for the bits of fp32 vectors that bf16 pieces cannot hold."""
import numpy as np
import pytest

from oracle import q4 as oq4
from test_gpu_mx4 import check_product, random_mx4
from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def whole(sq, torch, rows, cols, seed):  # noqa: F811
    """A matrix of multiples of 1/2 up to 6, exponents 127."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.randint(-(1 << 31), (1 << 31) - 1, (rows, 4 * (-(-cols // 32))), generator=g,
                          device="cuda", dtype=torch.int64).to(torch.int32)
    words[:, -(-cols // 8):] = 0
    scale = torch.full((rows, -(-cols // 32)), 127, dtype=torch.uint8, device="cuda")
    return sq.Mx4Weights(words, scale, rows, cols)


def small(torch, n, cols, seed, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, (n, cols), generator=g, device="cuda").to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("nvec,cols", [(1, 8), (5, 8), (40, 40), (7, 520), (20, 520)])
def test_more_rows_than_a_launch(sq, torch, nvec, cols, dtype):  # noqa: F811
    rows = (1 << 21) + 37 if cols < 100 else (1 << 21) + 3
    q = whole(sq, torch, rows, cols, 1)
    x = small(torch, nvec, cols, 2, dtype)
    y = sq.mx4_gemv(q, x, torch.float32)
    ref = x.float() @ sq.mx4_dequantize(q).t()
    assert torch.equal(y, ref)


@pytest.mark.parametrize("na,nb,cols", [(3, (1 << 21) + 37, 40), (3, (1 << 21) + 37, 520), (70, (1 << 21) + 5, 8),
                                        (33000, 70, 72), (33000, 300, 520), (40000, 5, 1032),
                                        (300, 33005, 512), (257, 65600, 520), (129, 200, 768)])
def test_more_coded_rows_than_a_launch(sq, torch, na, nb, cols):  # noqa: F811
    a, b = whole(sq, torch, na, cols, 3), whole(sq, torch, nb, cols, 4)
    y = sq.mx4_matmul(a, b)
    ref = sq.mx4_dequantize(a) @ sq.mx4_dequantize(b).t()
    assert torch.equal(y, ref)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_more_vectors_than_a_pass(sq, torch, dtype):  # noqa: F811
    q = whole(sq, torch, 70, 136, 5)
    x = small(torch, 32768 + 19, 136, 6, dtype)
    assert torch.equal(sq.mx4_gemv(q, x, torch.float32), x.float() @ sq.mx4_dequantize(q).t())


@pytest.mark.parametrize("dtype,nvec", [("bfloat16", 1), ("float16", 3), ("float32", 3), ("bfloat16", 9)])
def test_long_rows(sq, torch, dtype, nvec):  # noqa: F811
    cols = (1 << 22) + 4104
    q = whole(sq, torch, 2, cols, 7)
    x = torch.zeros(nvec, cols, dtype=getattr(torch, dtype), device="cuda")
    at = torch.randint(cols, (nvec, 3000), generator=torch.Generator().manual_seed(1)).cuda()
    x.scatter_(1, at, 1.0)
    x[:, -1] = 2.0
    y = sq.mx4_gemv(q, x, torch.float32)
    W = sq.mx4_dequantize(q)
    ref = torch.stack([(x[v].float() * W).sum(1) for v in range(nvec)])
    assert torch.equal(y, ref)
    b = sq.mx4_matmul(sq.mx4_quantize(x), q)
    codes = sq.mx4_dequantize(sq.mx4_quantize(x))
    assert torch.equal(b, torch.stack([(codes[v] * W).sum(1) for v in range(nvec)]))


@pytest.mark.parametrize("nvec", [1, 6, 40])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -112, 2.0 ** -100, 2.0 ** 110])
def test_vectors_of_fp32_at_the_ends_of_the_range(sq, torch, nvec, size):  # noqa: F811
    rng = np.random.default_rng(nvec)
    q, W = random_mx4(sq, torch, rng, 70, 520, 126, 130)
    x = (rng.uniform(-1, 1, (nvec, 520)) * size).astype(np.float32)
    y = sq.mx4_gemv(q, torch.from_numpy(x).cuda()).double().cpu().numpy()
    x = x.astype(np.float64)
    lost = 2.0 ** -133 * np.abs(W).sum(1) if size < 1 else 0.0
    exact, mag = x @ W.T, np.abs(x) @ np.abs(W).T
    assert np.all(np.abs(y - exact) <= (48 + 520 / 8) * 2.0 ** -24 * mag + lost + 2.0 ** -149)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("nvec", [1, 6, 40])
def test_the_largest_and_smallest_16_bit_vectors(sq, torch, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(nvec)
    q, W = random_mx4(sq, torch, rng, 70, 520, 100, 104)
    dt = getattr(torch, dtype)
    for v in (torch.finfo(dt).max / 16, torch.finfo(dt).smallest_normal / 4):
        x = (torch.from_numpy(rng.choice([-1.0, 0.5, 0.25], (nvec, 520))) * v).to(dt)
        y = sq.mx4_gemv(q, x.cuda(), torch.float32)
        if dtype == "bfloat16" and v < 1:    # products among fp32's subnormals: whole steps of 2^-149
            err = np.abs(y.double().cpu().numpy() - x.double().numpy() @ W.T)
            assert np.all(err <= 520 * 2.0 ** -149)
        else:
            check_product(y, x.double().numpy(), W, "float32")


def test_padding_behind_the_last_column_of_a_vector_product(sq, torch):  # noqa: F811
    # codes behind the last column are not weights of a product with vectors, whatever they are
    rng = np.random.default_rng(2)
    q, W = random_mx4(sq, torch, rng, 70, 520)
    for nvec in (1, 6, 40):
        x = torch.from_numpy(rng.normal(0, 1, (nvec, 520))).bfloat16().cuda()
        ref = sq.mx4_gemv(q, x)
        dirty = sq.Mx4Weights(q.codes.clone(), q.scale, 70, 520)
        dirty.codes[:, 65:] = 0x7F1E2D3C
        assert torch.equal(sq.mx4_gemv(dirty, x), ref)
    assert oq4.row_words(520) == q.codes.shape[1] == 68
