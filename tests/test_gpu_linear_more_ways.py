"""Backward passes that take the ways which the lists of test_gpu_linear_plans.py leave out: dX in shares of every tile and by the
kernels for few rows, dW in tiles of each size, whole and in shares."""
import pytest

from tests import test_gpu_linear_plans as lists

SHAPES = [(9906, 348, 3), (74, 2432, 8192), (1, 1920, 8704), (1, 1, 6592), (17130, 78, 3648), (207, 9088, 6528), (3, 576, 6080),
          (7000, 32, 64), (1, 1216, 6080), (1, 1536, 8384), (570, 74, 8896), (10141, 1, 2368), (19050, 4672, 70), (8197, 9280, 148)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape):
    lists.test_backward("bf16", shape)
