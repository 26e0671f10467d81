"""The backward of a dropped element: its gradient is 0 whatever its pre-activation and its dY held, as in the forward."""
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.test_gpu_linear import CODES, make


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(40, 100, 60), (200, 128, 256)])
def test_a_dropped_pre_activation_may_hold_anything(shape, dt, act, bad):
    M, K, N = shape
    X, W, _, _, Z, dY = make(M, K, N, ref.DTYPES[dt], 51, False, False)
    rng = ref.rng_tensor(5, 6, "cuda")
    kw = dict(activation=CODES[act], dropout=0.5, rng=rng)
    dropped = torch.from_numpy(ref.multiplier(M, N, 0.5, 5, 6, 0)).cuda() == 0
    want = mhffn.linear_backward(X, W, dY, Z, **kw)
    fill = torch.full_like(Z, bad)
    got = mhffn.linear_backward(X, W, torch.where(dropped, fill, dY), torch.where(dropped, fill, Z), **kw)
    assert all(torch.equal(got[k], want[k]) for k in want)
