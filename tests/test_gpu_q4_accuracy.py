"""How near products of coded normal weights come to 64 bits, in fp32 and fp16, for vectors
of both signs and of one sign.

Bar: 2.5e-7 of the result's 2-norm. Where the zero point is off the codes before they are
multiplied, a group of 128 is eight additions to a running sum that grows like a random
walk: each errs by at most 2^-23 of the sum (a truncated one, rms 0.42 x 2^-23), so
together by sqrt(1/8 + .. + 8/8) = 2.1 times that, 1.1e-7 of the group's sum, and the sum over
G <= 64 groups by sqrt(G / 2) 0.42 x 2^-24, up to 1.4e-7 more: 1.8e-7 for independent errors. The sign
of x does not enter, as the weights have both. Sums that keep the zero point, or that add the
pieces of an fp32 vector to one sum, pass the bar by a factor of 1.5 to 13 at these sizes."""
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("sign", ["both", "one"])
@pytest.mark.parametrize("rows,cols,nvec,group,zeros", [
    (1024, 4096, 64, 128, False), (1024, 4096, 64, 128, True), (1000, 8192, 20, 512, True),
    (1001, 4096, 130, 64, False), (512, 520, 512, 256, False), (1500, 4104, 33, 128, True),
    (33000, 264, 300, 128, True), (1024, 4096, 12, 128, True), (1024, 4096, 2, 128, False)])
def test_products_within_a_few_roundings(sq, torch, rows, cols, nvec, group, zeros, sign, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + nvec)
    q = sq.q4_quantize(torch.randn(rows, cols, device="cuda", generator=g) * 0.02, group, zeros=zeros)
    x = torch.randn(nvec, cols, device="cuda", generator=g).to(getattr(torch, dtype))
    if sign == "one":
        x = x.abs()
    exact = x.double() @ sq.q4_dequantize(q).double().t().contiguous()
    err = (sq.q4_gemv(q, x, torch.float32).double() - exact).norm() / exact.norm()
    assert err.item() <= 2.5e-7, err.item()


def test_every_code_and_zero_point(sq, torch):
    # u - z of every pair, by a vector that is 1 in one column: s (u - z) exactly, one piece
    # of the vector at a time too
    rows, cols = 256, 64
    u = torch.arange(256, device="cuda") % 16
    z = torch.arange(256, device="cuda") // 16
    words = torch.zeros(rows, 8, dtype=torch.int64, device="cuda")
    for i in range(8):
        words |= (u[:, None] << (4 * i))
    codes = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    scale = torch.full((rows, 2), 0.5, dtype=torch.float16, device="cuda")
    q = sq.Q4Weights(codes, scale, z[:, None].expand(rows, 2).to(torch.uint8).contiguous(), rows, cols, 32)
    ref = 0.5 * (u - z).float()
    for value in (1.0, 2.0 ** -9, 1.0 + 2.0 ** -9 + 2.0 ** -18):
        x = torch.zeros(cols, cols, device="cuda")
        x.fill_diagonal_(value)
        y = sq.q4_gemv(q, x, torch.float32)
        assert torch.equal(y, (ref * value).expand(cols, rows))
