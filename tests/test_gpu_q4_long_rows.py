"""Products with rows of 2^31 columns and more: every way of a product, by whole numbers
whose sums are exact in any order."""
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu

COLS = (1 << 31) + 136
NVEC = 17


def test_product_of_a_row_past_2_31_columns(sq, torch):
    words = sq.seedq_q4_row_words(COLS)
    need = COLS // 2 + 2 * NVEC * COLS + sq.seedq_q4_gemv_workspace_bytes(1, COLS, NVEC, 2)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip(f"{need >> 30} GiB of device memory wanted")
    codes = torch.full((1, words), -2004318072, dtype=torch.int32, device="cuda")   # 0x88888888: zero
    codes[0, COLS // 8:] = 0
    for at in (0, (1 << 28) - 1, (1 << 28) + 1, COLS // 8 - 1):
        codes[0, at] = -1717986919                                                  # 0x99999999: one
    scale = torch.full((1, -(-COLS // 128)), 0.5, dtype=torch.float16, device="cuda")
    q = sq.Q4Weights(codes, scale, None, 1, COLS, 128)
    x = torch.empty((NVEC, COLS), dtype=torch.bfloat16, device="cuda")
    for v in range(NVEC):
        x[v] = v + 1
    for nvec in (1, 3, NVEC):
        y = sq.q4_gemv(q, x[:nvec], torch.float32)
        assert y[:, 0].tolist() == [4 * 8 * 0.5 * (v + 1) for v in range(nvec)]
    del x, codes, scale, q, y
    torch.cuda.empty_cache()
