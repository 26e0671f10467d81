"""Dropout alone against its definition; captured steps that draw new masks; streams; the module
with its residual branch; and the operators together as a layer uses them."""
import numpy as np
import pytest
import torch

from paper_2512_06989_amd import mhffn
from tests import linear_reference as ref
from tests.helpers import TOL

SEED, OFFSET, CALL = 77, 2 ** 40, 2 ** 63


def normal(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (3, 7), (5, 9), (64, 16), (333, 1001), (1000, 264), (4097, 3), (2, 70001)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0, 2.0 ** -16, 1 - 2.0 ** -16])
def test_against_the_definition(shape, p, dt):
    dtype = ref.DTYPES[dt]
    X, R = normal(1, *shape, dtype=dtype), normal(2, *shape, dtype=dtype)
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    mult = ref.multiplier(*shape, p, SEED, OFFSET, CALL)
    for residual in (None, R):
        got = mhffn.dropout(X, p, rng, call=CALL, residual=residual)
        want = ref.f64(X) * mult
        error = 2 * ref.U2 * np.abs(want)
        if residual is not None:
            want = want + ref.f64(R)
            error = error + ref.U2 * np.abs(want)
        ref.check(got, want, ref.half_step(dtype) * np.abs(want) + 2 * error, TOL[dt], "%s %s" % (shape, p))
        if residual is None:   # exactly which stay
            assert np.array_equal(ref.f64(mhffn.dropout(torch.ones_like(X), p, rng, call=CALL)) != 0, mult != 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_strides_and_in_place(dt):
    dtype, M, N = ref.DTYPES[dt], 50, 75
    X, R = normal(3, M, N, dtype=dtype), normal(4, M, N, dtype=dtype)
    rng = ref.rng_tensor(1, 2, "cuda")
    want = mhffn.dropout(X, 0.3, rng, residual=R)
    for extra in (5, 8):
        wide = torch.full((3, M, N + extra), float("nan"), dtype=dtype, device="cuda")
        x, r, y = (wide[i, :, :N] if (M * (N + extra) * wide.element_size() * i) % 16 == 0 else None for i in range(3))
        if None in (x, r, y):
            x, r, y = (torch.full((M, N + extra), float("nan"), dtype=dtype, device="cuda")[:, :N] for _ in range(3))
        x.copy_(X)
        r.copy_(R)
        assert torch.equal(mhffn.dropout(x, 0.3, rng, residual=r, out=y), want)
        assert torch.equal(y, want)
    x, r = X.clone(), R.clone()
    assert mhffn.dropout(x, 0.3, rng, residual=R, out=x) is not None and torch.equal(x, want)
    mhffn.dropout(X, 0.3, rng, residual=r, out=r)
    assert torch.equal(r, want)
    assert mhffn.dropout(X[:0], 0.3, rng).shape == (0, N)


@pytest.mark.gpu
def test_what_is_dropped_is_zero_whatever_it_held():
    X = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0] * 500, device="cuda").reshape(20, 100)
    rng = ref.rng_tensor(8, 9, "cuda")
    kept = ref.multiplier(20, 100, 0.5, 8, 9, 0) != 0
    got = mhffn.dropout(X, 0.5, rng).cpu().numpy()
    assert np.all(got[~kept] == 0) and np.array_equal(np.isnan(got), np.isnan(X.cpu().numpy()) & kept)
    assert torch.all(mhffn.dropout(X, 1.0, rng) == 0)


@pytest.mark.gpu
def test_more_elements_than_32_bits_count():
    """More than 2^32 elements, and more than 2^32 rows of one element each (a piece of the mask per row)."""
    rng = ref.rng_tensor(SEED, OFFSET, "cuda")
    for M, N in ((65600, 65544), (2 ** 32 + 300, 1)):
        X = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
        mhffn.dropout(X, 0.25, rng, call=1, out=X)
        for first, rows in ((0, 2), (M // 2, 2), (M - 200, 200)):
            mult = ref.multiplier(rows, N, 0.25, SEED, OFFSET, 1, first_row=first)
            got = ref.f64(X[first:first + rows])
            assert np.array_equal(got != 0, mult != 0)
        del X
        torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dt,shape", [("bf16", (300, 256, 384)), ("bf16", (16, 1024, 256)), ("bf16", (100, 75, 50)),
                                      ("f32", (300, 100, 60))])
def test_a_captured_step_draws_new_masks(dt, shape):
    """Forward, backward and dropout in a graph; the offset advances between replays, eager work runs
    in between, every replay gives the eager result of its offset."""
    M, K, N = shape
    dtype = ref.DTYPES[dt]
    X, W, b, R = normal(5, M, K, dtype=dtype), normal(6, K, N, dtype=dtype, scale=K ** -0.5), normal(7, N, dtype=dtype), normal(8, M, N, dtype=dtype)
    rng = ref.rng_tensor(SEED, 0, "cuda")

    def step():
        Y, Z = mhffn.linear_forward(X, W, b, R, activation=mhffn.ACT_GELU, dropout=0.2, rng=rng, call=0, save=True)
        D = mhffn.dropout(Y, 0.1, rng, call=1)
        dY = mhffn.dropout(D, 0.1, rng, call=1)
        g = mhffn.linear_backward(X, W, dY, Z, activation=mhffn.ACT_GELU, dropout=0.2, rng=rng, call=0)
        return [Y, Z, D, *g.values()]

    mhffn.init()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    seen = []
    for replay in range(4):
        rng[1] = 10 * replay
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), replay
        seen.append(got[0])
    assert not any(torch.equal(seen[0], s) for s in seen[1:])


@pytest.mark.gpu
def test_two_streams_at_once():
    M, K, N = 500, 512, 515
    X, W = normal(9, M, K), normal(10, K, N, scale=K ** -0.5)
    dY, rng = normal(11, M, N), ref.rng_tensor(1, 2, "cuda")
    kw = dict(dropout=0.1, rng=rng)
    want_y, want = mhffn.linear_forward(X, W, **kw), mhffn.linear_backward(X, W, dY, **kw)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(8):
        for s in streams:
            got.append((mhffn.linear_forward(X, W, stream=s, **kw), mhffn.linear_backward(X, W, dY, stream=s, **kw)))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want_y) and all(torch.equal(g[k], want[k]) for k in want) for y, g in got)


def _module(N, H, dh, dtype, seed=1):
    dm, std = H * dh, 0.05
    t = [normal(seed, N, dm, dtype=dtype), normal(seed + 1, dm, dm, dtype=dtype, scale=dm ** -0.5)]
    t += [normal(seed + 2 + i, H, 3, 64, dh, dtype=dtype, scale=std) for i in range(3)]
    return t + [normal(seed + 5, H, dh, 3, dtype=dtype, scale=std), normal(seed + 6, dm, dm, dtype=dtype, scale=dm ** -0.5)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 16, 200, 1500])
@pytest.mark.parametrize("dropout", [0.0, 0.1])
def test_the_module_with_its_residual_branch(N, dropout, dt):
    """O, Q, S and the gradients are those of the parts: the module, the linear layer, dropout."""
    dtype = ref.DTYPES[dt]
    X, Wi, Wg, Wu, Wd, Wr, Wo = _module(N, 2, 128, dtype)
    R, dO, rng = normal(20, N, 256, dtype=dtype), normal(21, N, 256, dtype=dtype), ref.rng_tensor(SEED, OFFSET, "cuda")
    kw = dict(dropout=dropout, rng=rng, call=4)
    O, Q, S = mhffn.module_forward(X, Wi, Wg, Wu, Wd, Wr, Wo, residual=R, **kw)
    o, q, s = mhffn.module_forward(X, Wi, Wg, Wu, Wd, Wr, Wo)
    assert torch.equal(Q, q) and torch.equal(S, s)
    assert torch.equal(O, mhffn.linear_forward(S, Wo, None, R, **kw))
    mult = ref.multiplier(N, 256, dropout, SEED, OFFSET, 4)
    y, ey, _, _ = ref.forward(ref.f64(S), ref.f64(Wo), None, ref.f64(R), "none", mult, dtype)
    ref.check(O, y, ey, TOL[dt], "O")
    got = mhffn.module_backward(X, Wi, Wg, Wu, Wd, Wr, Wo, Q, S, dO, **kw)
    want = mhffn.module_backward(X, Wi, Wg, Wu, Wd, Wr, Wo, Q, S, mhffn.dropout(dO, dropout, rng, call=4))
    assert all(torch.equal(got[k], want[k]) for k in mhffn.MODULE_GRADS)
    if dropout:   # without a residual; the residual in place, rows apart, is X itself
        only = mhffn.module_forward(X, Wi, Wg, Wu, Wd, Wr, Wo, **kw)[0]
        assert torch.equal(only, mhffn.linear_forward(S, Wo, **kw))
    wide = torch.full((N, 256 + 24), 7.0, dtype=dtype, device="cuda")
    stream_rows = wide[:, :256]
    stream_rows.copy_(X)
    mhffn.module_forward(X, Wi, Wg, Wu, Wd, Wr, Wo, residual=stream_rows, out={"O": stream_rows}, **kw)
    assert torch.equal(stream_rows, mhffn.linear_forward(S, Wo, None, X, **kw)) and torch.all(wide[:, 256:] == 7.0)
    assert mhffn.module_forward(X[:0], Wi, Wg, Wu, Wd, Wr, Wo, residual=R[:0], **kw)[0].shape == (0, 256)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_layer_of_them(dt):
    """A model's layer: an input projection with bias, the module on the residual stream, a dense FFN
    with its residual and dropout; forward and backward, against 64 bits stage by stage."""
    dtype, N, dm, ff = ref.DTYPES[dt], 120, 256, 352
    X, Wi, Wg, Wu, Wd, Wr, Wo = _module(N, 2, 128, dtype, seed=30)
    W0, b0 = normal(40, dm, dm, dtype=dtype, scale=dm ** -0.5), normal(41, dm, dtype=dtype)
    W1, b1 = normal(42, dm, ff, dtype=dtype, scale=dm ** -0.5), normal(43, ff, dtype=dtype)
    W2, b2 = normal(44, ff, dm, dtype=dtype, scale=ff ** -0.5), normal(45, dm, dtype=dtype)
    rng, d = ref.rng_tensor(3, 5, "cuda"), dict(dropout=0.1, rng=ref.rng_tensor(3, 5, "cuda"))
    h0 = mhffn.linear_forward(X, W0, b0)
    h1, Q, S = mhffn.module_forward(h0, Wi, Wg, Wu, Wd, Wr, Wo, residual=h0, call=0, **d)
    u, Z = mhffn.linear_forward(h1, W1, b1, activation=mhffn.ACT_GELU, save=True)
    h2 = mhffn.linear_forward(u, W2, b2, h1, call=1, **d)
    f = ref.f64
    m1 = ref.multiplier(N, dm, 0.1, 3, 5, 1)
    for got, args in ((h0, (X, W0, b0, None, "none", 1.0)), (u, (h1, W1, b1, None, "gelu", 1.0)), (h2, (u, W2, b2, h1, "none", m1))):
        y, e, _, _ = ref.forward(*(f(t) for t in args[:4]), args[4], args[5], dtype)
        ref.check(got, y, e, TOL[dt])
    dh2 = normal(46, N, dm, dtype=dtype)
    g2 = mhffn.linear_backward(u, W2, dh2, call=1, **d)
    g1 = mhffn.linear_backward(h1, W1, g2["dX"], Z, activation=mhffn.ACT_GELU)
    dh1 = mhffn.dropout(g1["dX"], 0.0, rng, residual=dh2)
    gm = mhffn.module_backward(h0, Wi, Wg, Wu, Wd, Wr, Wo, Q, S, dh1, call=0, **d)
    dh0 = mhffn.dropout(gm["dX"], 0.0, None, residual=dh1)
    g0 = mhffn.linear_backward(X, W0, dh0)
    for got, args in ((g2, (u, W2, None, dh2, "none", m1)), (g1, (h1, W1, Z, g2["dX"], "gelu", np.ones((N, ff)))),
                      (g0, (X, W0, None, dh0, "none", np.ones((N, dm))))):
        want = ref.backward(*(f(t) for t in args[:4]), args[4], args[5], dtype)
        for k, (v, e) in want.items():
            ref.check(got[k], v, e, TOL[dt], k)
    ref.check(dh1, f(g1["dX"]) + f(dh2), ref.half_step(dtype) * np.abs(f(g1["dX"]) + f(dh2)) + ref.U2 * np.abs(f(dh2)), TOL[dt])
