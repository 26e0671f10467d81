"""Activations and their slopes at infinite pre-activations: the limits.  A pre-activation that overflowed may not turn its
row of dX, its column of dW and its sum in db into NaN.  NaN stays NaN."""
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.test_gpu_linear import CODES

INF = float("inf")
#               act(inf), act(-inf), act'(inf), act'(-inf)
LIMITS = {"none": (INF, -INF, 1.0, 1.0), "relu": (INF, 0.0, 1.0, 0.0), "silu": (INF, 0.0, 1.0, 0.0), "gelu": (INF, 0.0, 1.0, 0.0)}


@pytest.mark.gpu
@pytest.mark.parametrize("act", list(LIMITS))
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 40, 700])
def test_infinite_pre_activations(M, act, dt):
    dtype, K, N = ref.DTYPES[dt], 64, 96
    X, W = torch.zeros(M, K, dtype=dtype, device="cuda"), torch.zeros(K, N, dtype=dtype, device="cuda")
    bias = torch.zeros(N, dtype=dtype, device="cuda")
    bias[5], bias[40], bias[77] = INF, -INF, float("nan")
    Y, Z = mhffn.linear_forward(X, W, bias, activation=CODES[act], save=True)
    up, down, slope_up, slope_down = LIMITS[act]
    assert torch.all(Y[:, 5] == up) and torch.all(Y[:, 40] == down) and torch.all(torch.isnan(Y[:, 77]))
    assert torch.all(Z[:, 5] == INF) and torch.all(Z[:, 40] == -INF) and torch.all(torch.isnan(Z[:, 77]))
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[[5, 40, 77]] = False
    assert torch.all(Y[:, rest] == 0)
    Z[:, 77] = 0
    ones = torch.ones_like(Y)
    g = mhffn.linear_backward(torch.ones_like(X), torch.ones_like(W), ones, Z, activation=CODES[act])
    assert torch.all(g["dbias"][5] == M * slope_up) and torch.all(g["dbias"][40] == M * slope_down)
    assert torch.all(g["dW"][:, 5] == M * slope_up) and torch.all(g["dW"][:, 40] == M * slope_down)
    assert all(torch.all(torch.isfinite(t)) for t in g.values())
    if act not in ("none", "relu"):     # (relu's slope is a comparison)
        Z[:, 77] = float("nan")
        g = mhffn.linear_backward(torch.ones_like(X), torch.ones_like(W), ones, Z, activation=CODES[act])
        assert torch.isnan(g["dbias"][77]) and torch.all(torch.isfinite(g["dbias"][rest]))
