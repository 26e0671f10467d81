"""GELU in fp32 relative to its own value, where that is small: for negative z, 1 + erf(z / sqrt(2)) cancels.

u = 2^-24.  Phi(z) = erfc(a) / 2 of a = -z / sqrt(2), whose constant and product are rounded: |da / a| <= 2 u.  erfc moves by
a erfc'(a) / erfc(a) <= 2 a^2 + 1 = z^2 + 1 times that, and the library's erfc is good to 16 ulp = 32 u.  So Phi is within
(z^2 + 17) 2 u of itself, z Phi within one u more.  The density 2^(-z^2 log2(e) / 2) has three roundings in its exponent (3/2 z^2 u
in its value), one ulp of the instruction and three roundings around it."""
import math

import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref

U2 = ref.U2
LEAST = 2.0 ** -120      # (numbers below 2^-126 may be flushed, times |z|)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 70])
def test_relative_error(M):
    z = np.float32(np.concatenate([np.linspace(-13, 13, 2081), -np.geomspace(1e-6, 12.5, 400), np.geomspace(1e-6, 12.5, 400)]))
    N = len(z)
    bias = torch.from_numpy(z).cuda()
    X, W = torch.zeros(M, 8, device="cuda"), torch.zeros(8, N, device="cuda")
    Y, Z = mhffn.linear_forward(X, W, bias, activation=mhffn.ACT_GELU, save=True)
    assert torch.equal(Z, bias.expand(M, N))
    x = z.astype(np.float64)
    phi = np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    Phi = 0.5 * torch.special.erfc(torch.from_numpy(-x / math.sqrt(2))).numpy()
    off, most = np.abs(ref.f64(Y) - x * Phi), np.abs(x * Phi) * (x * x + 18) * U2 + LEAST
    assert np.all(off <= most), (x[np.argmax((off / most)[0])], np.max(off / most))
    g = mhffn.linear_backward(X[:1], W, torch.ones(1, N, device="cuda"), Z[:1], activation=mhffn.ACT_GELU, want=("dbias",))
    want = Phi + x * phi
    off, most = np.abs(ref.f64(g["dbias"]) - want), U2 * ((x * x + 17) * Phi + (x * x + 4) * np.abs(x) * phi + np.abs(want)) + LEAST
    assert np.all(off <= most), (x[np.argmax(off / most)], np.max(off / most))
