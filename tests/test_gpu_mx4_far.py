"""Products of microscaled 4-bit floats whose blocks lie far apart while all of them count: the
vectors' columns (the other matrix's exponents) undo the blocks' exponents, so that an exponent
applied to a wrong block changes every output. The bars are those of test_gpu_mx4."""
import numpy as np
import pytest

from oracle import mx4 as omx
from oracle import q4 as oq4
from test_gpu_mx4 import check_product
from test_gpu_q4 import TYPES, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def far_mx4(sq, torch, rng, rows, cols, exponents):  # noqa: F811
    """Random codes; a block's exponents lie around its own one of `exponents`."""
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    scale = (exponents + rng.integers(-2, 3, (rows, len(exponents)))).astype(np.uint8)
    words = torch.from_numpy(oq4.pack(codes).view(np.int32)).cuda()
    return sq.Mx4Weights(words, torch.from_numpy(scale).cuda(), rows, cols), omx.values(codes, scale)


# the ways: few vectors, batches, tiles, with columns in one and in several parts
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nvec", [1, 2, 4, 6, 11, 24, 40, 150])
@pytest.mark.parametrize("rows,cols", [(40, 520), (70, 4104), (1030, 264), (9, 72)])
def test_gemv(sq, torch, rows, cols, nvec, dtype):  # noqa: F811
    rng = np.random.default_rng(rows + nvec)
    reach = 10 if dtype == "float16" else 60    # fp16 holds 2^-10 .. 2^10 of a normal number
    exponents = 127 + rng.integers(-reach, reach + 1, -(-cols // 32))
    q, W = far_mx4(sq, torch, rng, rows, cols, exponents)
    x = rng.normal(0, 1, (nvec, cols)) * np.ldexp(1.0, 127 - exponents)[np.arange(cols) // 32]
    x = torch.from_numpy(x).to(getattr(torch, dtype))
    check_product(sq.mx4_gemv(q, x.cuda(), torch.float32), x.double().numpy(), W, "float32")


# few rows, tiles of 128 (short rows, whole and not) and of 256
@pytest.mark.parametrize("na,nb,cols", [(1, 70, 520), (5, 300, 4104), (20, 70, 520), (40, 300, 1032), (64, 1001, 2056),
                                        (130, 300, 264), (7, 90, 72), (300, 500, 520), (256, 384, 512),
                                        (130, 260, 8200), (4100, 4100, 520), (4096, 4096, 768)])
def test_matmul(sq, torch, na, nb, cols):  # noqa: F811
    rng = np.random.default_rng(na + nb)
    exponents = 127 + rng.integers(-60, 61, -(-cols // 32))
    a, A = far_mx4(sq, torch, rng, na, cols, exponents)
    b, B = far_mx4(sq, torch, rng, nb, cols, 254 - exponents)
    check_product(sq.mx4_matmul(a, b), A, B, "float32")
