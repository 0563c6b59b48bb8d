"""Products of vectors near both ends of fp32's range: what the weights' own products
s (u - z) x and their sums hold, the products straight from the codes hold too.

The vectors are normal, cut at 3.9, times 2^e. At e = 125 they reach 0.97 x 2^127, where a
sum of u x over a few columns already passes fp32's largest value, while s (u - z) has an
rms of at most 0.041 (codes and zero points 0 .. 15, scales up to 0.006), so that sums of
1032 terms have an rms of at most 1.3 x 2^125 and stay below 2^128 at 6 deviations. At
e = -90 a vector's three 8-bit pieces reach down to 2^-133 for elements from 2^-110 on,
2^-20 of the rest. Bars: those of the middle of the range."""
import numpy as np
import pytest

from test_gpu_q4 import _check_product, _random_q4, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (512, False)])
@pytest.mark.parametrize("nvec", [1, 2, 3, 8, 40, 200])
@pytest.mark.parametrize("e", [-90, 125])
def test_vectors_at_the_ends_of_the_range(sq, torch, nvec, group, zeros, dtype, e):
    rng = np.random.default_rng(nvec + group)
    q, W = _random_q4(sq, torch, rng, 70, 1032, group, zeros)
    x = np.clip(rng.normal(0, 1, (nvec, 1032)), -3.9, 3.9) * 2.0 ** e
    x = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype))
    exact = x.double().numpy() @ W.T
    assert np.abs(exact).max() < 2.0 ** 127
    _check_product(sq.q4_gemv(q, x.cuda(), torch.float32), exact, "float32")


@pytest.mark.parametrize("nvec", [1, 3, 40])
def test_one_signed_vectors_at_the_largest_value(sq, torch, nvec):
    # every x the largest bf16, codes 9 on zero point 8 in a few columns: y is a few x
    rows, cols = 33, 520
    big = torch.finfo(torch.bfloat16).max
    codes = torch.full((rows, sq.seedq_q4_row_words(cols)), -2004318072, dtype=torch.int32, device="cuda")
    codes[:, 7] = -1717986919                        # 0x99999999: one
    codes[:, cols // 8:] = 0
    scale = torch.full((rows, -(-cols // 128)), 2.0 ** -6, dtype=torch.float16, device="cuda")
    q = sq.Q4Weights(codes, scale, None, rows, cols, 128)
    for dt in (torch.bfloat16, torch.float32):
        x = torch.full((nvec, cols), big, dtype=dt, device="cuda")
        assert (sq.q4_gemv(q, x, torch.float32) == big / 8).all()
