"""The module with its residual branch at other widths, heads and row strides: the parts' results, and the output projection
against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL
from tests.test_gpu_dropout import OFFSET, SEED, _module, normal


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 17, 333, 2100])
@pytest.mark.parametrize("H,dh", [(1, 64), (3, 64), (5, 64), (3, 128), (8, 128), (1, 256), (3, 256)])
def test_widths_and_strides(H, dh, N, dt):
    dtype, dm = ref.DTYPES[dt], H * dh
    X, *W = _module(N, H, dh, dtype, seed=80)
    R, dO, rng = normal(90, N, dm, dtype=dtype), normal(91, N, dm, dtype=dtype), ref.rng_tensor(SEED, OFFSET, "cuda")
    kw = dict(dropout=0.2, rng=rng, call=7)
    strided = lambda t, extra: torch.cat([t, torch.full((N, extra), 7.0, dtype=dtype, device="cuda")], 1)[:, :dm]  # noqa: E731
    out = strided(torch.zeros_like(X), 16)
    O, Q, S = mhffn.module_forward(strided(X, 8), *W, residual=strided(R, 24), out={"O": out}, **kw)
    _, q, s = mhffn.module_forward(X, *W)
    assert O.data_ptr() == out.data_ptr() and torch.equal(Q, q) and torch.equal(S, s)
    assert torch.equal(O, mhffn.module_forward(X, *W, residual=R, **kw)[0])
    mult = ref.multiplier(N, dm, 0.2, SEED, OFFSET, 7)
    y, ey, _, _ = ref.forward(ref.f64(S), ref.f64(W[-1]), None, ref.f64(R), "none", mult, dtype)
    ref.check(O, y, ey, TOL[dt], "O")
    got = mhffn.module_backward(X, *W, Q, S, strided(dO, 32), **kw)
    want = mhffn.module_backward(X, *W, Q, S, mhffn.dropout(dO, 0.2, rng, call=7))
    assert all(torch.equal(got[k], want[k]) for k in mhffn.MODULE_GRADS)
    # a dropped element of dO is nothing, whatever it holds
    bad = torch.where(torch.from_numpy(np.asarray(mult) == 0).cuda(), torch.full_like(dO, float("nan")), dO)
    got = mhffn.module_backward(X, *W, Q, S, bad, **kw)
    assert all(torch.equal(got[k], want[k]) for k in mhffn.MODULE_GRADS)
