"""The linear layer with its epilogue against the definition in 64 bits: every element within the bound
of its own roundings (tests/linear_reference.py), the whole within the library's Frobenius bound."""
import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL

CODES = {"none": mhffn.ACT_NONE, "relu": mhffn.ACT_RELU, "silu": mhffn.ACT_SILU, "gelu": mhffn.ACT_GELU}
SEED, OFFSET, CALL = 2 ** 63 + 12345, 2 ** 32 - 2, 9

# rows, d_in, d_out: single rows and columns, below and around tile edges, nothing that divides
# anything, contractions shorter and longer than a slice, many rows, wide and narrow
SHAPES = [(1, 1, 1), (1, 64, 64), (1, 2048, 80), (2, 3, 1), (3, 8, 8), (5, 7, 9), (8, 1000, 16), (16, 192, 80),
          (17, 33, 31), (31, 4099, 5), (33, 128, 96), (64, 32, 40), (65, 96, 2049), (100, 64, 1500), (129, 40, 1000),
          (130, 96, 72), (257, 128, 264), (300, 1001, 515), (511, 520, 130), (1000, 1024, 256), (2050, 64, 64)]
# activation, dropout, bias, residual, Z kept
EPILOGUES = [("none", 0.0, False, False, False), ("none", 0.1, True, True, False), ("relu", 0.25, True, False, True),
             ("silu", 0.0, False, True, True), ("gelu", 0.5, True, True, True), ("gelu", 0.0, True, False, False),
             ("silu", 0.1, True, True, False), ("relu", 1.0, False, True, True)]


def make(M, K, N, dtype, seed, bias, residual):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    return (n(M, K), n(K, N, scale=K ** -0.5), n(N) if bias else None, n(M, N) if residual else None, n(M, N), n(M, N))


def check_forward(M, K, N, dt, epilogue, seed=1):
    name, p, bias, residual, keep = epilogue
    dtype = ref.DTYPES[dt]
    X, W, b, R, _, _ = make(M, K, N, dtype, seed, bias, residual)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    got = mhffn.linear_forward(X, W, b, R, activation=CODES[name], dropout=p, rng=rng, call=CALL, save=keep)
    mult = ref.multiplier(M, N, p, SEED, OFFSET, CALL)
    Y, eY, Z, eZ = ref.forward(ref.f64(X), ref.f64(W), ref.f64(b), ref.f64(R), name, mult, dtype)
    what = "%s %s %s" % ((M, K, N), dt, epilogue)
    if keep:
        ref.check(got[1], Z, eZ, TOL[dt], what + " Z")
        got = got[0]
    ref.check(got, Y, eY, TOL[dt], what + " Y")


def check_backward(M, K, N, dt, epilogue, seed=1):
    name, p = epilogue[:2]
    dtype = ref.DTYPES[dt]
    X, W, _, _, Z, dY = make(M, K, N, dtype, seed, False, False)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    got = mhffn.linear_backward(X, W, dY, Z if name != "none" else None, activation=CODES[name], dropout=p, rng=rng,
                                call=CALL)
    mult = ref.multiplier(M, N, p, SEED, OFFSET, CALL)
    want = ref.backward(ref.f64(X), ref.f64(W), ref.f64(Z), ref.f64(dY), name, mult, dtype)
    assert set(got) == set(want)
    for k, (value, bound) in want.items():
        ref.check(got[k], value, bound, TOL[dt], "%s %s %s %s" % ((M, K, N), dt, epilogue, k))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward_shapes(i, dt):
    for j in (0, 3, 5):
        check_forward(*SHAPES[i], dt, EPILOGUES[(i + j) % len(EPILOGUES)])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward_shapes(i, dt):
    for j in (0, 3, 5):
        check_backward(*SHAPES[i], dt, EPILOGUES[(i + j) % len(EPILOGUES)])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("shape", [(7, 256, 128), (150, 128, 136), (70, 50, 203)])
def test_every_epilogue(shape, epilogue, dt):
    check_forward(*shape, dt, epilogue, seed=2)
    check_backward(*shape, dt, epilogue, seed=2)


def strided(t, extra, fill):
    """`t` in rows that lie `extra` elements further apart, everything around them set to `fill`."""
    M, N = t.shape
    wide = torch.full((M + 2, N + extra), fill, dtype=t.dtype, device=t.device)
    base = wide.view(-1)[8:]          # (16-byte aligned, not at the start of the allocation)
    rows = base.as_strided((M, N), (N + extra, 1))
    rows.copy_(t)
    return wide, rows


def around(wide, rows):
    """Everything of `wide` that is not in `rows`."""
    mask = torch.ones_like(wide, dtype=torch.bool)
    mask.view(-1)[8:].as_strided(rows.shape, rows.stride()).fill_(False)
    return wide[mask]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [8, 24, 1, 13])
@pytest.mark.parametrize("shape", [(37, 64, 96), (5, 2048, 64), (200, 75, 50), (300, 256, 384)])
def test_row_strides(shape, extra, dt):
    """Strided rows give the bits of dense ones, nothing between them is read (NaN) or written."""
    M, K, N = shape
    X, W, b, R, Z, dY = make(M, K, N, ref.DTYPES[dt], 4, True, True)
    rng = ref.rng_tensor(3, 4, "cuda")
    kw = dict(activation=mhffn.ACT_GELU, dropout=0.2, rng=rng, call=1)
    Y, Zk = mhffn.linear_forward(X, W, b, R, save=True, **kw)
    grads = mhffn.linear_backward(X, W, dY, Zk, **kw)
    _, Xs = strided(X, extra, float("nan"))
    _, Rs = strided(R, extra + 2, float("nan"))
    _, dYs = strided(dY, extra + 3, float("nan"))
    wide_y, Ys = strided(torch.zeros_like(Y), extra + 1, 7.0)
    wide_x, dXs = strided(torch.zeros_like(X), extra, 7.0)
    Z2 = torch.zeros_like(Zk)
    got = mhffn.linear_forward(Xs, W, b, Rs, save=True, out={"Y": Ys, "Z": Z2}, **kw)
    assert got[0].data_ptr() == Ys.data_ptr() and got[1] is not None
    assert torch.equal(Ys, Y) and torch.equal(Z2, Zk) and torch.all(around(wide_y, Ys) == 7.0)
    g = mhffn.linear_backward(Xs, W, dYs, Zk, out={"dX": dXs}, **kw)
    assert torch.equal(dXs, grads["dX"]) and torch.all(around(wide_x, dXs) == 7.0)
    assert torch.equal(g["dW"], grads["dW"]) and torch.equal(g["dbias"], grads["dbias"])
    assert mhffn.linear_backward(Xs, W, dYs, Zk, **kw)["dX"].stride(0) == Xs.stride(0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(9, 256, 128), (100, 75, 51), (400, 256, 384)])
def test_outputs_stay_within_their_tensors(shape, dt):
    """Every output between guard bands in one buffer; the residual in place."""
    M, K, N = shape
    dtype = ref.DTYPES[dt]
    X, W, b, R, Z, dY = make(M, K, N, dtype, 5, True, True)
    want = mhffn.linear_forward(X, W, b, R, activation=mhffn.ACT_SILU, save=True)
    grads = mhffn.linear_backward(X, W, dY, want[1], activation=mhffn.ACT_SILU)
    ups = lambda n: (n + 63) // 64 * 64  # noqa: E731
    sizes = {"Y": (M, N), "Z": (M, N), "dX": (M, K), "dW": (K, N), "dbias": (N,)}
    buffer = torch.full((sum(ups(int(np.prod(s))) + 64 for s in sizes.values()) + 64,), 7.0, dtype=dtype, device="cuda")
    views, at, used = {}, 64, torch.zeros_like(buffer, dtype=torch.bool)
    for k, s in sizes.items():
        n = int(np.prod(s))
        views[k] = buffer[at:at + n].view(s)
        used[at:at + n] = True
        at += ups(n) + 64
    views["Y"].copy_(R)
    mhffn.linear_forward(X, W, b, views["Y"], activation=mhffn.ACT_SILU, save=True, out={"Y": views["Y"], "Z": views["Z"]})
    mhffn.linear_backward(X, W, dY, views["Z"], activation=mhffn.ACT_SILU, out={k: views[k] for k in ("dX", "dW", "dbias")})
    assert torch.equal(views["Y"], want[0]) and torch.equal(views["Z"], want[1])
    for k in grads:
        assert torch.equal(views[k], grads[k]), k
    assert torch.all(buffer[~used] == 7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_some_gradients_alone(dt):
    X, W, _, _, Z, dY = make(90, 64, 100, ref.DTYPES[dt], 6, False, False)
    for act in (mhffn.ACT_NONE, mhffn.ACT_GELU):
        every = mhffn.linear_backward(X, W, dY, Z, activation=act)
        for want in (("dX",), ("dW",), ("dbias",), ("dbias", "dX"), ()):
            got = mhffn.linear_backward(X, W, dY, Z, activation=act, want=want)
            assert set(got) == set(want) and all(torch.equal(got[k], every[k]) for k in want)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_no_rows(dt):
    X, W, b, R, Z, dY = make(0, 33, 21, ref.DTYPES[dt], 7, True, True)
    assert mhffn.linear_forward(X, W, b, R).shape == (0, 21)
    out = {"dW": torch.full_like(W, 7.0), "dbias": torch.full_like(b, 7.0)}
    g = mhffn.linear_backward(X, W, dY, Z, activation=mhffn.ACT_RELU, out=out)
    assert g["dX"].shape == (0, 33) and torch.all(g["dW"] == 0) and torch.all(g["dbias"] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(40, 100, 60), (40, 128, 64), (200, 128, 256), (300, 1001, 515)])
def test_infinities_and_nan_stay_in_their_rows(shape, dt):
    """A row of X that holds NaN gives a row of NaN and leaves the others' bits; padding and clamped
    rows of a tile bring nothing in.  A dropped element is 0 whatever it held."""
    M, K, N = shape
    X, W, b, R, Z, dY = make(M, K, N, ref.DTYPES[dt], 8, True, True)
    want = mhffn.linear_forward(X, W, b, R)
    bad = X.clone()
    bad[M - 1] = float("nan")
    bad[0, K - 1] = float("inf")
    got = mhffn.linear_forward(bad, W, b, R)
    assert torch.equal(got[1:M - 1], want[1:M - 1])
    assert torch.all(torch.isnan(got[M - 1])) and not torch.any(torch.isfinite(got[0]))
    rng = ref.rng_tensor(5, 6, "cuda")
    mult = torch.from_numpy(ref.multiplier(M, N, 0.5, 5, 6, 0)).cuda()
    got = mhffn.linear_forward(bad, W, b, R, dropout=0.5, rng=rng)
    assert torch.equal(got[M - 1][mult[M - 1] == 0], R[M - 1][mult[M - 1] == 0])
    assert torch.all(torch.isnan(got[M - 1][mult[M - 1] != 0]))
    bad_dy = torch.where(mult == 0, torch.full_like(dY, float("nan")), dY)
    a, c = (mhffn.linear_backward(X, W, g, dropout=0.5, rng=rng) for g in (bad_dy, dY))
    assert all(torch.equal(a[k], c[k]) for k in a)
    bad_w = W.clone()
    bad_w[:, N - 1] = float("nan")
    got = mhffn.linear_forward(X, bad_w, b, R)
    assert torch.equal(got[:, :N - 1], want[:, :N - 1]) and torch.all(torch.isnan(got[:, N - 1]))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_activations_far_from_zero(act, dt):
    """Z = X through the identity: values of every size, both signs, and what the limits give."""
    values = [0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 0.7, -0.7, 3.0, -3.0, 5.5, -5.5, 9.0, -9.0, 20.0, -20.0, 90.0,
              -90.0, 300.0, -300.0, 1e10, -1e10, 1e30, -1e30, 2.5, -2.5, 12.5, -12.5, 1.0, -1.0, 4.0, -4.0]
    dtype = ref.DTYPES[dt]
    X = torch.tensor(values, dtype=dtype, device="cuda").reshape(1, 32)
    I = torch.eye(32, dtype=dtype, device="cuda")
    x = ref.f64(X)
    Y = mhffn.linear_forward(X, I, activation=CODES[act])
    with np.errstate(over="ignore"):
        want, rate = ref.act(x, act), ref.slope(x, act)
    # (the function's own error shrinks with its value for positive z and is absolute for negative ones)
    bound = ref.half_step(dtype) * np.abs(want) + 2 * ref.FN * np.maximum(np.abs(want), 1) + 34 * ref.U2 * np.abs(x) * (x > -100)
    assert np.all(np.abs(ref.f64(Y) - want) <= bound)
    ones = torch.ones_like(X)
    g = ref.f64(mhffn.linear_backward(X, I, ones, X, activation=CODES[act], want=("dX",))["dX"])
    assert np.all(np.abs(g - rate) <= 2 * ref.half_step(dtype) * np.abs(rate) + 4 * ref.FN)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_the_same_bits_every_time(dt):
    for shape in ((16, 2048, 512), (1000, 1024, 256), (3000, 200, 333)):
        X, W, b, R, Z, dY = make(*shape, ref.DTYPES[dt], 9, True, True)
        rng = ref.rng_tensor(1, 1, "cuda")
        runs = []
        for _ in range(2):
            y = mhffn.linear_forward(X, W, b, R, activation=mhffn.ACT_SILU, dropout=0.1, rng=rng)
            g = mhffn.linear_backward(X, W, dY, Z, activation=mhffn.ACT_SILU, dropout=0.1, rng=rng)
            runs.append([y, *g.values()])
        assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Rows that lie so far apart that X, Y and dX span more than 2^32 elements."""
    M, K, N, ld = 70000, 64, 72, 1 << 16
    X, W, b, _, Z, dY = make(M, K, N, torch.bfloat16, 10, True, False)
    wide = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    Xs = wide.as_strided((M, K), (ld, 1))
    Ys = wide.as_strided((M, N), (ld, 1), 1 << 14)
    dXs = wide.as_strided((M, K), (ld, 1), 1 << 15)
    Xs.copy_(X)
    want = mhffn.linear_forward(X, W, b)
    mhffn.linear_forward(Xs, W, b, out={"Y": Ys})
    assert torch.equal(Ys, want)
    grads = mhffn.linear_backward(X, W, want)
    got = mhffn.linear_backward(Xs, W, Ys, out={"dX": dXs})
    assert torch.equal(dXs, grads["dX"]) and torch.equal(got["dW"], grads["dW"]) and torch.equal(got["dbias"], grads["dbias"])


@pytest.mark.gpu
def test_large_training_shapes_on_sampled_rows():
    """The shapes of a training batch: sampled rows of Y, Z and dX, sampled columns of dW."""
    M, K, N = 16384, 2048, 5632
    X, W, b, _, Z, dY = make(M, K, N, torch.bfloat16, 11, True, False)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    kw = dict(activation=mhffn.ACT_GELU, dropout=0.1, rng=rng, call=CALL)
    Y, Zk = mhffn.linear_forward(X, W, b, save=True, **kw)
    g = mhffn.linear_backward(X, W, dY, Z, **kw)
    rows = torch.tensor([0, 1, 255, 256, 8191, 9000, M - 2, M - 1])
    mult = np.concatenate([ref.multiplier(1, N, 0.1, SEED, OFFSET, CALL, first_row=int(r)) for r in rows])
    wx = ref.f64(W)
    y, ey, z, ez = ref.forward(ref.f64(X[rows]), wx, ref.f64(b), None, "gelu", mult, torch.bfloat16)
    ref.check(Y[rows], y, ey, 5e-3, "Y")
    ref.check(Zk[rows], z, ez, 5e-3, "Z")
    want = ref.backward(ref.f64(X[rows]), wx, ref.f64(Z[rows]), ref.f64(dY[rows]), "gelu", mult, torch.bfloat16)
    ref.check(g["dX"][rows], *want["dX"], 5e-3, "dX")
    cols = torch.tensor([0, 1, 255, 256, 3000, N - 1])
    full = ref.multiplier(M, N, 0.1, SEED, OFFSET, CALL)[:, cols]
    want = ref.backward(ref.f64(X), wx[:, cols], ref.f64(Z[:, cols]), ref.f64(dY[:, cols]), "gelu", full, torch.bfloat16)
    ref.check(g["dW"][:, cols], *want["dW"], 5e-3, "dW")
    ref.check(g["dbias"][cols], *want["dbias"], 5e-3, "dbias")
