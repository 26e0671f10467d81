"""The scale of the dropout in a backward.  Without an activation or with relu, an element of dZ is dY's times 0 or the scale: held
back until the sums, the scale costs no rounding, and the gradients are rounded once, like sums over the kept elements of dY."""
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.test_gpu_linear import CALL, CODES, OFFSET, SEED, make


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
# few rows, a shared launch, tiles one after the other, shares of the contraction, widths that nothing divides
@pytest.mark.parametrize("shape", [(16, 64, 64), (300, 256, 384), (2048, 2048, 512), (4111, 520, 1032), (333, 101, 51)])
def test_rounded_once(shape, dt, act):
    M, K, N = shape
    dtype, h = ref.DTYPES[dt], ref.half_step(ref.DTYPES[dt])
    X, W, _, _, Z, dY = make(M, K, N, dtype, 61, False, False)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    got = mhffn.linear_backward(X, W, dY, Z, activation=CODES[act], dropout=0.1, rng=rng, call=CALL)
    mult = torch.from_numpy(ref.multiplier(M, N, 0.1, SEED, OFFSET, CALL)).cuda()
    x, w, dz = X.double(), W.double(), dY.double() * mult
    if act == "relu":
        dz = torch.where(Z.double() > 0, dz, 0.0)
    # sums of n products in fp32, in any order (n + 2) 2 u of their magnitudes, then the scale and the storage type
    for k, want, size, n in (("dX", dz @ w.t().contiguous(), dz.abs() @ w.t().contiguous().abs(), N),
                             ("dW", x.t().contiguous() @ dz, x.t().contiguous().abs() @ dz.abs(), M),
                             ("dbias", dz.sum(0), dz.abs().sum(0), M)):
        bound = h * want.abs() + (1 + h) * (n + 3) * ref.U2 * size
        ref.check(got[k], ref.f64(want), ref.f64(bound), 1.0, "%s %s" % (k, shape))
        if dt == "bf16" and want.numel() >= 4096:
            # An error of one rounding is uniform within a half step of its binade: h / sqrt(3) of the binade's lower end, on
            # average over magnitudes 0.425 h of the value; of two roundings 0.60 h.  4096 of them scatter by 1 %.
            off = (got[k].double() - want).norm() / want.norm()
            assert off < 0.48 * h, (k, float(off / h))
