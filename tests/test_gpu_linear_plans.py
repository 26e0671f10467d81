"""The linear layer at sizes that reach each of its tiles, splits of the contraction and shared launches,
in every form, against the definition in 64 bits on sampled rows and columns."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL
from tests.test_gpu_linear import CALL, CODES, OFFSET, SEED, make

# rows, d_in, d_out; contractions of odd numbers of 32, rows and widths past a tile's edge
FORWARD = [("bf16", s) for s in (
    (5, 96, 40), (5, 2080, 40), (5, 512, 515), (5, 40, 40), (5, 4128, 4104), (100, 2048, 1024), (1000, 544, 2000),
    (1030, 4128, 515), (2000, 2080, 2000), (2050, 512, 515), (2050, 4128, 1032), (3000, 96, 1032), (3000, 512, 2056),
    (3000, 200, 4104), (4100, 4128, 72), (4100, 32, 4104), (6200, 96, 2056), (6200, 512, 136))] + [("f32", s) for s in (
    (5, 512, 40), (4100, 40, 515), (4100, 1056, 72), (1500, 515, 1001), (2000, 768, 2048))]
BACKWARD = [("bf16", s) for s in (
    (5, 40, 4104), (5, 4128, 4104), (1000, 1024, 1024), (4100, 96, 40), (4111, 520, 1032), (6200, 200, 1032),
    (6200, 200, 2056), (6200, 512, 72), (6200, 1056, 515), (6200, 2080, 264), (6200, 4128, 264), (6223, 2080, 4104))
] + [("f32", s) for s in ((5, 40, 515), (100, 4128, 4104), (520, 40, 40), (1030, 40, 515), (1500, 1001, 515), (4100, 4128, 72))]


def plan(op, dt, shape):
    lib = mhffn.load()
    d = mhffn.LinearDesc(*shape, 0, 0, 0, 1 if dt == "bf16" else 0, CODES["gelu"], 0.1, 0)
    text = ctypes.create_string_buffer(256)
    lib.mhffn_linear_plan_text(ctypes.byref(d), op, text, 256)
    return text.value.decode()


def test_the_sizes_take_different_ways():
    ways = {plan(8, *c) for c in FORWARD} | {plan(9, *c) for c in BACKWARD}
    assert "" not in ways and len(ways) > 20


def test_rows_that_no_launch_could_count():
    lib = mhffn.load()
    for rows, works in ((2 ** 28, True), (2 ** 28 + 1, False), (2 ** 40, False)):
        d = mhffn.LinearDesc(rows, 33, 8, 0, 0, 0, 1, 0, 0.0, 0)
        for op in (8, 9):
            assert (lib.mhffn_linear_workspace_bytes(ctypes.byref(d), op) > 0) == works


def some(n, most=96):
    """Up to `most` indices below n: both ends, the edges of tiles, an odd step between."""
    edges = {i for e in (64, 128, 256, n) for i in (e - 1, e, n // e * e, n // e * e - 1)} | {0, n - 1}
    return torch.tensor(sorted(i for i in edges | set(range(7, n, max(1, n // most) | 1)) if 0 <= i < n))


def empty(*shape, dtype):
    """Memory that gives itself away where nothing is stored"""
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("dt,shape", FORWARD)
def test_forward(dt, shape):
    M, K, N = shape
    dtype = ref.DTYPES[dt]
    X, W, b, R, _, _ = make(M, K, N, dtype, 21, True, True)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    out = {"Y": empty(M, N, dtype=dtype), "Z": empty(M, N, dtype=dtype)}
    Y, Z = mhffn.linear_forward(X, W, b, R, activation=mhffn.ACT_GELU, dropout=0.1, rng=rng, call=CALL, save=True, out=out)
    assert torch.all(torch.isfinite(Y)) and torch.all(torch.isfinite(Z))
    rows = some(M)
    mult = np.concatenate([ref.multiplier(1, N, 0.1, SEED, OFFSET, CALL, first_row=int(r)) for r in rows])
    y, ey, z, ez = ref.forward(ref.f64(X[rows]), ref.f64(W), ref.f64(b), ref.f64(R[rows]), "gelu", mult, dtype)
    ref.check(Z[rows], z, ez, TOL[dt], "Z")
    ref.check(Y[rows], y, ey, TOL[dt], "Y")


@pytest.mark.gpu
@pytest.mark.parametrize("dt,shape", BACKWARD)
def test_backward(dt, shape):
    M, K, N = shape
    dtype = ref.DTYPES[dt]
    X, W, _, _, Z, dY = make(M, K, N, dtype, 22, False, False)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    kw = dict(activation=mhffn.ACT_GELU, dropout=0.1, rng=rng, call=CALL)
    out = {"dX": empty(M, K, dtype=dtype), "dW": empty(K, N, dtype=dtype), "dbias": empty(N, dtype=dtype)}
    g = mhffn.linear_backward(X, W, dY, Z, out=out, **kw)
    assert all(torch.all(torch.isfinite(t)) for t in g.values())
    for k in g:   # each gradient alone has the bits that it has among the others
        assert torch.equal(mhffn.linear_backward(X, W, dY, Z, want=(k,), **kw)[k], g[k]), k
    w = ref.f64(W)
    rows, cols = some(M), some(N)
    mult = np.concatenate([ref.multiplier(1, N, 0.1, SEED, OFFSET, CALL, first_row=int(r)) for r in rows])
    want = ref.backward(ref.f64(X[rows]), w, ref.f64(Z[rows]), ref.f64(dY[rows]), "gelu", mult, dtype)
    ref.check(g["dX"][rows], *want["dX"], TOL[dt], "dX")
    mult = ref.multiplier(M, N, 0.1, SEED, OFFSET, CALL)[:, cols]
    want = ref.backward(ref.f64(X), w[:, cols], ref.f64(Z[:, cols]), ref.f64(dY[:, cols]), "gelu", mult, dtype)
    ref.check(g["dW"][:, cols], *want["dW"], TOL[dt], "dW")
    ref.check(g["dbias"][cols], *want["dbias"], TOL[dt], "dbias")


@pytest.mark.gpu
@pytest.mark.parametrize("dt,shape", [("bf16", (70, 96, 64)), ("bf16", (33, 2080, 40)), ("bf16", (5, 4128, 4104)), ("bf16", (3000, 96, 1032)),
                                      ("bf16", (6200, 96, 2056)), ("f32", (70, 97, 64)), ("f32", (5, 512, 40))])
def test_an_infinity_anywhere_along_the_contraction(dt, shape):
    """One infinite k of row 0: the row is infinite with W's signs, wherever shares and slices end, and no
    other row's bits move."""
    M, K, N = shape
    X, W, b, _, _, _ = make(M, K, N, ref.DTYPES[dt], 23, True, False)
    want = mhffn.linear_forward(X, W, b)
    signs = torch.where(W == 0, torch.full_like(W, float("nan")), W * float("inf"))
    for k in {0, 31, 32, 63, 64, K // 2, K - 33, K - 32, K - 1}:
        bad = X.clone()
        bad[0, k] = float("inf")
        got = mhffn.linear_forward(bad, W, b)
        assert torch.equal(got[1:], want[1:]), k
        assert torch.equal(got[0].nan_to_num(7.0, 1e30, -1e30), signs[k].nan_to_num(7.0, 1e30, -1e30)), k


@pytest.mark.gpu
@pytest.mark.parametrize("dt,shape", [("bf16", (33, 64, 64)), ("bf16", (1001, 128, 96)), ("bf16", (4111, 520, 1032)), ("bf16", (6223, 2080, 264)),
                                      ("f32", (33, 64, 64)), ("f32", (1501, 101, 51))])
def test_an_infinite_token(dt, shape):
    """One infinite element of X makes its row of dW infinite with dY's signs, the other rows keep their bits:
    also in the last tokens, after which a slice of the contraction holds none."""
    M, K, N = shape
    X, W, _, _, _, dY = make(M, K, N, ref.DTYPES[dt], 24, False, False)
    want = mhffn.linear_backward(X, W, dY, want=("dW",))["dW"]
    signs = torch.where(dY == 0, torch.full_like(dY, float("nan")), dY * float("inf"))
    for m in {0, M // 2, M - 33, M - 2, M - 1}:
        bad = X.clone()
        bad[m, 3] = float("inf")
        got = mhffn.linear_backward(bad, W, dY, want=("dW",))["dW"]
        assert torch.equal(got[3].nan_to_num(7.0, 1e30, -1e30), signs[m].nan_to_num(7.0, 1e30, -1e30)), m
        got[3] = want[3]
        assert torch.equal(got, want), m


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("ld", [(1 << 22) - 8, 1 << 22, (1 << 22) + 8, (1 << 23) + 40])
def test_rows_that_lie_far_apart(ld, dt):
    M, K, N = 70, 96, 72
    X, W, b, R, _, dY = make(M, K, N, ref.DTYPES[dt], 25, True, True)
    far = torch.full((M * ld,), float("nan"), dtype=ref.DTYPES[dt], device="cuda")
    at = [far.as_strided((M, n), (ld, 1), 4096 * i) for i, n in enumerate((K, N, N, N, K))]
    for to, t in zip(at, (X, R, dY)):
        to.copy_(t)
    want = mhffn.linear_forward(X, W, b, R)
    assert torch.equal(mhffn.linear_forward(at[0], W, b, at[1], out={"Y": at[3]}), want)
    want = mhffn.linear_backward(X, W, dY)
    got = mhffn.linear_backward(at[0], W, at[2], out={"dX": at[4]})
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.gpu
def test_a_captured_step_of_every_launch():
    """Forward and backward at sizes that share a launch, split and pack, captured once and replayed on new inputs
    with other work between the replays."""
    shapes = [("bf16", (1000, 1024, 1024)), ("bf16", (333, 1001, 515)), ("bf16", (4111, 520, 1032)), ("f32", (1500, 1001, 515))]
    rng = ref.rng_tensor(3, 0, "cuda")
    kw = dict(activation=mhffn.ACT_SILU, dropout=0.1, rng=rng)
    for i, (dt, s) in enumerate(shapes):
        X, W, b, R, _, dY = make(*s, ref.DTYPES[dt], 26 + i, True, True)

        def step():
            y, z = mhffn.linear_forward(X, W, b, R, save=True, **kw)
            return [y, z, *mhffn.linear_backward(X, W, dY, z, **kw).values()]
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for r in range(3):
            X.mul_(-0.5)
            dY.mul_(0.75)
            rng[1] += 1
            graph.replay()
            want = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(got, want)), (dt, s, r)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 3, 16, 37])
@pytest.mark.parametrize("K", [8, 9, 31, 63, 64, 65, 100, 1001, 2063])
@pytest.mark.parametrize("N", [8, 9, 15, 16, 17, 23, 40, 515, 4101])
def test_a_few_rows_of_any_width(M, K, N):
    """Both ends of both operands in the middle of NaN, the residual in place, the columns around Y left alone."""
    X, W, b, R, _, _ = make(M, K, N, torch.bfloat16, 31, True, True)

    def among_nan(t, before=16):
        flat = torch.full((t.numel() + 64,), float("nan"), dtype=t.dtype, device="cuda")
        inside = flat[before:before + t.numel()].view(t.shape)
        inside.copy_(t)
        return inside
    wide = torch.full((M + 2, N + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = wide.view(-1)[16:].as_strided((M, N), (N + 5, 1))
    rows.copy_(R)
    xs = torch.full((M * (K + 3) + 32,), float("nan"), dtype=torch.bfloat16, device="cuda")
    Xs = xs[8:].as_strided((M, K), (K + 3, 1))
    Xs.copy_(X)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    mhffn.linear_forward(Xs, among_nan(W), among_nan(b), rows, activation=mhffn.ACT_SILU, dropout=0.1, rng=rng, call=CALL, out={"Y": rows})
    y, ey, _, _ = ref.forward(ref.f64(X), ref.f64(W), ref.f64(b), ref.f64(R), "silu", ref.multiplier(M, N, 0.1, SEED, OFFSET, CALL), torch.bfloat16)
    ref.check(rows, y, ey, TOL["bf16"], "Y")
    left = torch.ones_like(wide, dtype=torch.bool)
    left.view(-1)[16:].as_strided((M, N), (N + 5, 1)).fill_(False)
    assert torch.all(wide[left] == 7.0)
