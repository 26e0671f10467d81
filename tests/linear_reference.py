"""The linear layer with its epilogue and dropout in 64 bits, from their definition, with the
bounds that the GPU's results are held to.

Every bound counts roundings.  u = 2^-24 is fp32's half step, h = finfo(t).eps / 2 that of the
storage type t.  A sum of n products in fp32, in any order, is off by at most (n + 2) 2 u times the
sum of their magnitudes (2 u: the matrix instructions do not promise to round to nearest).  An
activation moves an error by at most its steepest slope (1.13) and adds its own: the library's
functions are good to a few u relative to their result and 2^-21 absolute relative to |z|."""
import math

import numpy as np
import torch

ACTS = ("none", "relu", "silu", "gelu")
U2 = 2.0 ** -23
STEEPEST = 1.13
FN = 2.0 ** -20      # an activation or its slope, evaluated in fp32: relative to max(|z|, 1)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def philox(piece, seed, step):
    """The four words of Philox4x32-10 for each piece: [len(piece), 4] uint32."""
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    piece = np.asarray(piece, dtype=np.uint64)
    c = [piece & low, piece >> s32, np.full_like(piece, step & 0xFFFFFFFF), np.full_like(piece, step >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> s32) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> s32) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).astype(np.uint32)


def threshold(p):
    return int(np.rint(np.float32(p) * np.float32(65536)))


def multiplier(rows, cols, p, seed, offset, call, first_row=0):
    """[rows, cols] float64: the scale where an element stays, 0 where it is dropped."""
    t = threshold(p)
    if t == 0:
        return np.ones((rows, cols))
    per = -(-cols // 8)
    piece = np.arange(first_row * per, (first_row + rows) * per, dtype=np.uint64)
    words = philox(piece, seed % 2 ** 64, (offset + call) % 2 ** 64)
    halves = words.astype("<u4").view("<u2").reshape(rows, 8 * per)[:, :cols]
    return (halves >= t) * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def rng_tensor(seed, offset, device):
    s = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v  # noqa: E731
    return torch.tensor([s(seed), s(offset)], dtype=torch.int64, device=device)


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "silu":
        return z / (1 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2))
    return z


def slope(z, name):
    if name == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def _erfc(x):
    return torch.special.erfc(torch.from_numpy(np.ascontiguousarray(x))).numpy()


def f64(t):
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def forward(X, W, bias, residual, name, mult, dtype):
    """(Y, bound of Y, Z, bound of Z), float64 arrays in and out."""
    h, K = half_step(dtype), X.shape[1]
    Z, size = X @ W, np.abs(X) @ np.abs(W)
    if bias is not None:
        Z, size = Z + bias, size + np.abs(bias)
    e = (K + 2) * U2 * size
    a = act(Z, name)
    Y, ea = mult * a, mult * (STEEPEST * e + (FN * np.maximum(np.abs(Z), 1) if name != "none" else 0) + U2 * np.abs(a))
    if residual is not None:
        Y = Y + residual
        ea = ea + U2 * np.abs(Y)
    return Y, h * np.abs(Y) + (1 + h) * ea, Z, h * np.abs(Z) + (1 + h) * e


def backward(X, W, Z, dY, name, mult, dtype):
    """{gradient: (value, bound)}; Z is the stored pre-activation.  dZ is rounded to the storage type
    where it is not dY itself."""
    h = half_step(dtype)
    M, N = dY.shape
    dZ = mult * dY * (1.0 if name == "none" else slope(Z, name))
    e = 3 * U2 * np.abs(dZ) + (0 if name == "none" else np.abs(mult * dY) * FN * np.maximum(np.abs(Z), 1))
    touched = name != "none" or not np.all(mult == 1.0)
    ez = e + (h * (np.abs(dZ) + e) if touched else 0)
    out = {}
    for key, value, size, error, n in (
            ("dX", dZ @ W.T, (np.abs(dZ) + ez) @ np.abs(W).T, ez @ np.abs(W).T, N),
            ("dW", X.T @ dZ, np.abs(X).T @ (np.abs(dZ) + ez), np.abs(X).T @ ez, M),
            ("dbias", dZ.sum(0), (np.abs(dZ) + e).sum(0), e.sum(0), M)):
        out[key] = (value, h * np.abs(value) + (1 + h) * ((n + 2) * U2 * size + error))
    return out


# The Frobenius figure is an average over roundings: one element may be off by two whole half steps of
# bf16 (dZ and the gradient), 2 * 2^-8 = 7.8e-3 > 5e-3.  Of 256 independent errors with a root mean square
# of 2 * 2^-8 / sqrt(3) / sqrt(2) = 3.2e-3 at most, the average scatters by 1 / sqrt(512) = 4 %.
AVERAGED = 256


def check(got, want, bound, frobenius, what=""):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want) - bound - 1e-38     # (a result may be a denormal number that is flushed)
    assert np.all(off <= 0), "%s: %d elements beyond their bound, the worst by %.3e of %.3e at %s" % (
        what, np.sum(~(off <= 0)), np.nanmax(off), bound.flat[np.nanargmax(off)], np.unravel_index(np.nanargmax(off), off.shape))
    norm = np.linalg.norm(want)
    if want.size < AVERAGED:
        return
    assert np.linalg.norm(got - want) <= frobenius * norm + 1e-30, "%s: %.3e" % (what, np.linalg.norm(got - want) / norm)
