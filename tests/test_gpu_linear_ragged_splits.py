"""The weight gradient in shares of the contraction where d_in is no multiple of 8: the product then has more rows
than dW, and each share's partial sums lie that many rows apart."""
import re

import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL
from tests.test_gpu_linear import CALL, OFFSET, SEED, make
from tests.test_gpu_linear_plans import empty, plan, some

# rows, d_in, d_out; d_in % 8 = 1, 3, 4, 7, 2, 5, 6; the last share of some is ragged
SHAPES = [(8192, 1001, 515), (16384, 515, 1001), (16384, 100, 200), (16384, 999, 72), (16383, 34, 40), (16384, 77, 520),
          (16001, 2046, 96)]


@pytest.mark.parametrize("shape", SHAPES)
def test_these_sizes_are_padded_and_shared_out(shape):
    way = plan(mhffn.OP_LINEAR_BACKWARD, "bf16", shape)
    assert shape[1] % 8 and "packed X" in way
    assert int(re.search(r"dW \d+x\d+ splits=(\d+)", way).group(1)) > 1, way


def test_every_rest_of_a_width_is_there():
    assert {s[1] % 8 for s in SHAPES} == {1, 2, 3, 4, 5, 6, 7}


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dt):
    M, K, N = shape
    dtype = ref.DTYPES[dt]
    X, W, _, _, Z, dY = make(M, K, N, dtype, 41, False, False)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    out = {"dX": empty(M, K, dtype=dtype), "dW": empty(K, N, dtype=dtype), "dbias": empty(N, dtype=dtype)}
    g = mhffn.linear_backward(X, W, dY, Z, activation=mhffn.ACT_SILU, dropout=0.1, rng=rng, call=CALL, out=out)
    rows, cols = some(M, 40), some(N, 40)
    mult = np.concatenate([ref.multiplier(1, N, 0.1, SEED, OFFSET, CALL, first_row=int(r)) for r in rows])
    w = ref.f64(W)
    want = ref.backward(ref.f64(X[rows]), w, ref.f64(Z[rows]), ref.f64(dY[rows]), "silu", mult, dtype)
    ref.check(g["dX"][rows], *want["dX"], TOL[dt], "dX")
    mult = ref.multiplier(M, N, 0.1, SEED, OFFSET, CALL)[:, cols]
    want = ref.backward(ref.f64(X), w[:, cols], ref.f64(Z[:, cols]), ref.f64(dY[:, cols]), "silu", mult, dtype)
    ref.check(g["dW"][:, cols], *want["dW"], TOL[dt], "dW")
    ref.check(g["dbias"][cols], *want["dbias"], TOL[dt], "dbias")


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_an_infinite_token(shape):
    """One infinite element of X makes its row of dW infinite with dY's signs and leaves the other rows' bits."""
    M, K, N = shape
    X, W, _, _, _, dY = make(M, K, N, torch.bfloat16, 42, False, False)
    want = mhffn.linear_backward(X, W, dY, want=("dW",))["dW"]
    signs = torch.where(dY == 0, torch.full_like(dY, float("nan")), dY * float("inf"))
    for m, k in ((0, 0), (M // 2, K // 2), (M - 33, 3), (M - 1, K - 1)):
        bad = X.clone()
        bad[m, k] = float("inf")
        got = mhffn.linear_backward(bad, W, dY, want=("dW",))["dW"]
        assert torch.equal(got[k].nan_to_num(7.0, 1e30, -1e30), signs[m].nan_to_num(7.0, 1e30, -1e30)), (m, k)
        got[k] = want[k]
        assert torch.equal(got, want), (m, k)
