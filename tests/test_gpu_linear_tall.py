"""Narrow layers of any height: the kernels for few rows are taken for one round of workgroups at most, whose row blocks a grid's
second dimension (65535) holds."""
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL
from tests.test_gpu_linear import make
from tests.test_gpu_linear_plans import plan

NARROW = [(k, n) for k in (64, 128, 192, 256, 1024) for n in (32, 64, 96, 128, 512)]


@pytest.mark.parametrize("M", [17, 300, 1024, 2048, 8192, 8193, 16384, 1 << 20, 1 << 21, (1 << 21) + 1, 3000000, 1 << 28])
def test_few_rows_are_few(M):
    for k, n in NARROW:
        one_round = (M + 31) // 32 * (n // 32) <= 256
        for op, shape in ((mhffn.OP_LINEAR_FORWARD, (M, k, n)), (mhffn.OP_LINEAR_BACKWARD, (M, n, k))):
            assert one_round or "few rows" not in plan(op, "bf16", shape), shape


def test_one_round_takes_them():
    assert plan(mhffn.OP_LINEAR_FORWARD, "bf16", (2048, 256, 64)) == plan(mhffn.OP_LINEAR_FORWARD, "bf16", (1, 2048, 2048)) == "few rows"


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [((1 << 21) + 100, 64, 32), ((1 << 21) + 100, 32, 64), (20000, 64, 96)])
def test_more_row_blocks_than_a_grid_is_high(shape):
    M, K, N = shape
    X, W, b, R, _, dY = make(M, K, N, torch.bfloat16, 71, True, True)
    Y = mhffn.linear_forward(X, W, b, R)
    g = mhffn.linear_backward(X, W, dY)
    rows = torch.cat([torch.arange(0, 40), torch.arange(M // 2, M // 2 + 40), torch.arange(M - 140, M)])
    y, ey, _, _ = ref.forward(ref.f64(X[rows]), ref.f64(W), ref.f64(b), ref.f64(R[rows]), "none", 1.0, torch.bfloat16)
    ref.check(Y[rows], y, ey, TOL["bf16"], "Y")
    want = ref.backward(ref.f64(X[rows]), ref.f64(W), None, ref.f64(dY[rows]), "none", 1.0, torch.bfloat16)
    ref.check(g["dX"][rows], *want["dX"], TOL["bf16"], "dX")
    x, d = X.double(), dY.double()
    dW, dbias = x.t().contiguous() @ d, d.sum(0)
    assert (g["dW"].double() - dW).norm() <= TOL["bf16"] * dW.norm()
    assert torch.all((g["dbias"].double() - dbias).abs() <= ref.half_step(torch.bfloat16) * dbias.abs() + 1.01 * M * ref.U2 * d.abs().sum(0))
