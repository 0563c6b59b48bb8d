"""Products in the forms that large matrices take, on random data: two tiles of rows a wave
(many vectors) or a workgroup (a batch), with several tiles of rows and vectors and
remainders of both, in every type and group size. Bars: those of test_gpu_q4.py."""
import functools

import numpy as np
import pytest

from test_gpu_q4 import TYPES, _check_product, _random_q4, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def matrix(sq, torch):
    # parameters of a matrix come in order, so each is made once
    return functools.lru_cache(maxsize=1)(lambda rows, cols, group, zeros: _random_q4(
        sq, torch, np.random.default_rng(rows + group), rows, cols, group, zeros))


def _product(sq, torch, matrix, rows, cols, nvec, group, zeros, dtype):
    q, W = matrix(rows, cols, group, zeros)
    rng = np.random.default_rng(nvec)
    x = torch.from_numpy(rng.normal(0, 1, (nvec, cols)).astype(np.float32)).to(getattr(torch, dtype))
    _check_product(sq.q4_gemv(q, x.cuda(), torch.float32), x.double().numpy() @ W.T, "float32")


# 65 tiles of 256 rows by 8 of 64 vectors
@pytest.mark.parametrize("group,zeros", [(32, True), (32, False), (64, True), (64, False), (128, True),
                                         (128, False), (256, True), (512, False)])
@pytest.mark.parametrize("dtype", TYPES)
def test_two_tiles_of_rows_a_wave(sq, torch, matrix, group, zeros, dtype):
    _product(sq, torch, matrix, 16424, 264, 500, group, zeros, dtype)


# 513 tiles of rows by one of 32 or 64 vectors
@pytest.mark.parametrize("group,zeros", [(32, True), (64, True), (128, False)])
@pytest.mark.parametrize("nvec", [20, 40])
@pytest.mark.parametrize("dtype", TYPES)
def test_two_tiles_of_rows_a_wave_and_few_vectors(sq, torch, matrix, group, zeros, nvec, dtype):
    _product(sq, torch, matrix, 131100, 136, nvec, group, zeros, dtype)


# 257 workgroups of 32 rows: a wave for each of the five blocks of columns (nine in groups of 32)
@pytest.mark.parametrize("group,zeros", [(32, True), (32, False), (64, True), (64, False), (128, True),
                                         (128, False), (256, True), (256, False), (512, True), (512, False)])
@pytest.mark.parametrize("nvec", [3, 9, 16])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_two_tiles_of_rows_a_workgroup(sq, torch, matrix, group, zeros, nvec, dtype):
    _product(sq, torch, matrix, 8200, 2056, nvec, group, zeros, dtype)


# 513 workgroups: four waves, the blocks divided unevenly
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (256, False)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_many_workgroups_of_a_batch(sq, torch, matrix, group, zeros, dtype):
    _product(sq, torch, matrix, 16400, 3080, 7, group, zeros, dtype)
