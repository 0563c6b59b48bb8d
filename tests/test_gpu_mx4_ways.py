"""Products of microscaled 4-bit floats at the borders of the ways that a product takes, with
the bars of test_gpu_mx4."""
import numpy as np
import pytest

from test_gpu_mx4 import check_product, random_mx4
from test_gpu_q4 import TYPES, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [8192, 8193, 16383, 16384, 16401])
@pytest.mark.parametrize("nvec", [1, 2, 3, 4])
def test_few_vectors_of_many_rows(sq, torch, rows, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(rows + nvec)
    for cols in (72, 520):
        q, W = random_mx4(sq, torch, rng, rows, cols)
        x = torch.from_numpy(rng.normal(0, 1, (nvec, cols))).to(getattr(torch, dtype))
        check_product(sq.mx4_gemv(q, x.cuda(), torch.float32), x.double().numpy(), W, "float32")


@pytest.mark.parametrize("nvec", [3, 4, 5, 6, 7, 8])
def test_few_vectors_of_very_long_rows(sq, torch, nvec):  # noqa: F811
    rng = np.random.default_rng(nvec)
    cols = (1 << 22) + 40
    q, W = random_mx4(sq, torch, rng, 3, cols)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32))
    check_product(sq.mx4_gemv(q, x.cuda()), x.double().numpy(), W, "float32")


# 5, 11 and 13 tiles of 32 vectors, and of fp32 3, 6, 9 and 15, each with few rows and with many
@pytest.mark.parametrize("rows,cols,nvec,dtype", [(300, 264, 160, "bfloat16"), (300, 264, 130, "float32"), (90, 1032, 340, "float16"),
                                                  (90, 1032, 416, "bfloat16"), (8000, 264, 416, "bfloat16"),
                                                  (8000, 264, 416, "float32"), (102500, 136, 96, "float32"),
                                                  (51300, 136, 192, "float32"), (34300, 264, 288, "float32"),
                                                  (20600, 520, 480, "float32"), (20600, 520, 470, "float16")])
def test_many_vectors_by_tiles(sq, torch, rows, cols, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(rows + nvec)
    q, W = random_mx4(sq, torch, rng, rows, cols)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols))).to(getattr(torch, dtype))
    check_product(sq.mx4_gemv(q, x.cuda(), torch.float32), x.double().numpy(), W, "float32")
