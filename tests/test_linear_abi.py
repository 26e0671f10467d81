"""Host-only tests of the linear layer and dropout: descriptors, refusals before any launch, scratch,
and what the Python binding says about wrong arguments."""
import ctypes
import os
import re

import pytest
import torch

from paper_2512_06989_amd import mhffn

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mhffn.h")).read()
FAKE = ctypes.c_void_p(0x10000)   # aligned, never dereferenced: validation fails first
OFF16, OFF8 = ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10004)


@pytest.mark.parametrize("name,cls", [("mhffn_linear_desc", mhffn.LinearDesc), ("mhffn_dropout_desc", mhffn.DropoutDesc)])
def test_descriptors_match_the_header(name, cls):
    body = HEADER[:HEADER.index("} %s;" % name)]
    body = body[body.rindex("typedef struct {"):]
    kinds = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float, "uint64_t": ctypes.c_uint64}
    fields = re.findall(r"^\s*(u?int64_t|int32_t|float)\s+(\w+);", body, re.M)
    assert [(n, kinds[t]) for t, n in fields] == cls._fields_


def linear(**kw):
    base = dict(n_rows=64, d_in=96, d_out=128, ld_x=0, ld_y=0, ld_r=0, dtype=mhffn.BF16, activation=0, dropout=0.0, call=0)
    base.update(kw)
    return mhffn.LinearDesc(*[base[f[0]] for f in mhffn.LinearDesc._fields_])


def drop(**kw):
    base = dict(n_rows=64, n_cols=96, ld_x=0, ld_y=0, ld_r=0, dtype=mhffn.BF16, dropout=0.1, call=0)
    base.update(kw)
    return mhffn.DropoutDesc(*[base[f[0]] for f in mhffn.DropoutDesc._fields_])


def fwd(d, ptrs=None, ws=None, size=0):
    return mhffn.load().mhffn_linear_forward(ctypes.byref(d), *(ptrs or [FAKE] * 7), ws, size, None)


def bwd(d, ptrs=None, ws=None, size=0):
    return mhffn.load().mhffn_linear_backward(ctypes.byref(d), *(ptrs or [FAKE] * 8), ws, size, None)


BAD = [(dict(n_rows=-1), 2), (dict(n_rows=(1 << 40) + 1), 2), (dict(d_in=0), 2), (dict(d_out=0), 2),
       (dict(d_in=(1 << 20) + 1), 2), (dict(d_out=(1 << 20) + 1), 2), (dict(ld_x=95), 2), (dict(ld_y=127), 2),
       (dict(ld_r=127), 2), (dict(dtype=2), 3), (dict(activation=4), 3), (dict(activation=-1), 3),
       (dict(dropout=-0.1), 2), (dict(dropout=1.5), 2), (dict(dropout=float("nan")), 2)]


@pytest.mark.parametrize("kw,status", BAD)
def test_linear_refuses_bad_descriptors(kw, status):
    assert fwd(linear(**kw), ws=FAKE, size=1 << 50) == status
    assert bwd(linear(**kw), ws=FAKE, size=1 << 50) == status
    for op in (mhffn.OP_LINEAR_FORWARD, mhffn.OP_LINEAR_BACKWARD):
        assert mhffn.load().mhffn_linear_workspace_bytes(ctypes.byref(linear(**kw)), op) == 0


def test_linear_refuses_missing_and_misaligned_pointers():
    d = linear(dropout=0.5, activation=mhffn.ACT_GELU)
    # X, W, bias, residual, rng, Y, Z
    for i, required in enumerate((True, True, False, False, True, True, False)):
        ptrs = [FAKE] * 7
        ptrs[i] = None
        if required:
            assert fwd(d, ptrs, FAKE, 1 << 50) == 1
        ptrs[i] = OFF8 if i == 4 else OFF16
        assert fwd(d, ptrs, FAKE, 1 << 50) == 4
    # X, W, Z, dY, rng, dX, dW, dbias
    for i, required in enumerate((True, True, True, True, True, False, False, False)):
        ptrs = [FAKE] * 8
        ptrs[i] = None
        if required:
            assert bwd(d, ptrs, FAKE, 1 << 50) == 1
        ptrs[i] = OFF8 if i == 4 else OFF16
        assert bwd(d, ptrs, FAKE, 1 << 50) == 4
    assert mhffn.load().mhffn_linear_forward(None, *([FAKE] * 7), None, 0, None) == 1
    assert mhffn.load().mhffn_linear_backward(None, *([FAKE] * 8), None, 0, None) == 1


@pytest.mark.parametrize("kw", [dict(d_in=100), dict(d_out=101, activation=1), dict(n_rows=5000, dropout=0.5),
                                dict(dtype=mhffn.F32, activation=2)])
def test_linear_refuses_a_small_or_misaligned_workspace(kw):
    d = linear(**kw)
    need = mhffn.load().mhffn_linear_workspace_bytes(ctypes.byref(d), mhffn.OP_LINEAR_BACKWARD)
    assert need > 0
    assert bwd(d, ws=None, size=need) == 5 and bwd(d, ws=FAKE, size=need - 1) == 5
    assert bwd(d, ws=ctypes.c_void_p(0x10010), size=need) == 4
    need = mhffn.load().mhffn_linear_workspace_bytes(ctypes.byref(d), mhffn.OP_LINEAR_FORWARD)
    if need:
        assert fwd(d, ws=None, size=need) == 5 and fwd(d, ws=FAKE, size=need - 1) == 5
        assert fwd(d, ws=ctypes.c_void_p(0x10010), size=need) == 4


def test_scratch_of_other_operations_is_none():
    for op in (0, 4, 7, 10, 99):
        assert mhffn.load().mhffn_linear_workspace_bytes(ctypes.byref(linear()), op) == 0


def test_no_rows():
    d = linear(n_rows=0, dropout=0.5, activation=2)
    for op in (mhffn.OP_LINEAR_FORWARD, mhffn.OP_LINEAR_BACKWARD):
        assert mhffn.load().mhffn_linear_workspace_bytes(ctypes.byref(d), op) == 0
    assert fwd(d, [None, FAKE, None, None, None, None, None]) == 0
    assert fwd(d, [None] * 7) == 1
    assert bwd(d, [None, FAKE, None, None, None, None, None, None]) == 0
    assert mhffn.load().mhffn_dropout(ctypes.byref(drop(n_rows=0)), None, None, None, None, None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(n_rows=-1), 2), (dict(n_cols=0), 2), (dict(n_cols=(1 << 20) + 1), 2), (dict(ld_x=95), 2), (dict(ld_y=95), 2),
    (dict(ld_r=95), 2), (dict(dtype=9), 3), (dict(dropout=1.01), 2), (dict(dropout=float("nan")), 2)])
def test_dropout_refuses_bad_descriptors(kw, status):
    assert mhffn.load().mhffn_dropout(ctypes.byref(drop(**kw)), *([FAKE] * 4), None) == status


def test_dropout_refuses_missing_and_misaligned_pointers():
    call = lambda *p: mhffn.load().mhffn_dropout(ctypes.byref(drop()), *p, None)  # noqa: E731
    assert mhffn.load().mhffn_dropout(None, FAKE, None, FAKE, FAKE, None) == 1
    assert call(None, None, FAKE, FAKE) == 1 and call(FAKE, None, FAKE, None) == 1 and call(FAKE, None, None, FAKE) == 1
    assert call(OFF16, None, FAKE, FAKE) == 4 and call(FAKE, OFF16, FAKE, FAKE) == 4
    assert call(FAKE, None, OFF8, FAKE) == 4 and call(FAKE, None, FAKE, OFF16) == 4


def module_desc(**kw):
    base = dict(n_tokens=64, n_heads=2, d_head=128, n_sub=3, d_sub=64, ld_x=0, ld_y=0, dtype=mhffn.BF16,
                route_mode=mhffn.ROUTE_PARAMS, eps=1e-6)
    base.update(kw)
    return mhffn.Desc(*[base[f[0]] for f in mhffn.Desc._fields_])


def residual_fwd(d, ptrs=None, ld=0, p=0.1, rng=FAKE, ws=FAKE, size=1 << 50):
    ptrs = ptrs or [FAKE] * 11     # X, seven weights, residual; O, Q, S
    return mhffn.load().mhffn_module_residual_forward(ctypes.byref(d), *ptrs[:8], ld, p, rng, 0, *ptrs[8:], ws, size, None)


def residual_bwd(d, ptrs=None, p=0.1, rng=FAKE, ws=FAKE, size=1 << 50):
    ptrs = ptrs or [FAKE] * 17     # X, six weights, Q, S, dO; seven gradients
    return mhffn.load().mhffn_module_residual_backward(ctypes.byref(d), *ptrs[:10], p, rng, 0, *ptrs[10:], ws, size, None)


def test_module_with_its_residual_branch_refuses():
    d = module_desc()
    assert residual_fwd(d, ld=255) == 2 and residual_fwd(d, p=2.0) == 2 and residual_bwd(d, p=-1.0) == 2
    assert residual_fwd(d, rng=None) == 1 and residual_bwd(d, rng=None) == 1
    assert residual_fwd(d, rng=OFF8) == 4 and residual_bwd(d, rng=OFF8) == 4
    for i in range(11):
        ptrs = [FAKE] * 11
        ptrs[i] = None
        if i != 7:
            assert residual_fwd(d, ptrs) == 1, i
        ptrs[i] = OFF16
        assert residual_fwd(d, ptrs) == 4, i
    for i in range(17):
        ptrs = [FAKE] * 17
        ptrs[i] = None
        if i < 10:
            assert residual_bwd(d, ptrs) == 1, i
        ptrs[i] = OFF16
        assert residual_bwd(d, ptrs) == 4, i
    weights = module_desc(route_mode=mhffn.ROUTE_WEIGHTS)
    assert residual_fwd(weights) == 3 and residual_bwd(weights) == 3
    for op, call in ((mhffn.OP_MODULE_RESIDUAL_FORWARD, residual_fwd), (mhffn.OP_MODULE_RESIDUAL_BACKWARD, residual_bwd)):
        need = mhffn.workspace_bytes(d, op)
        assert need > 0 and mhffn.workspace_bytes(weights, op) == 0
        assert call(d, size=need - 1) == 5 and call(d, ws=None) == 5 and call(d, ws=OFF16) == 4
    assert residual_fwd(module_desc(n_tokens=0), rng=None, ws=None) == 0


# ---- the Python binding: every case raises before the library is reached ---------------------
def _args(M=10, K=12, N=20, dtype=torch.bfloat16):
    return torch.zeros(M, K, dtype=dtype), torch.zeros(K, N, dtype=dtype)


@pytest.mark.parametrize("what,text", [
    ("w_shape", "W must have shape"), ("w_dtype", "W has dtype"), ("w_strided", "W must be contiguous"),
    ("x_strided", "X rows must be contiguous"), ("x_overlap", "X rows overlap"), ("x_vector", "X must be"),
    ("bias", "bias must have shape"), ("bias_dtype", "bias has dtype"), ("residual", "residual must be"),
    ("residual_dtype", "residual has dtype"), ("y", "Y must be"), ("z", "Z must be contiguous"),
    ("rng_dtype", "rng has dtype"), ("rng_shape", "rng must have shape"), ("p", "dropout must be"),
    ("call", "call must be"), ("device", "X is on cpu")])
def test_linear_forward_says_what_is_wrong(what, text):
    X, W = _args()
    kw = {}
    if what == "w_shape":
        W = torch.zeros(13, 20, dtype=torch.bfloat16)
    elif what == "w_dtype":
        W = W.float()
    elif what == "w_strided":
        W = torch.zeros(20, 12, dtype=torch.bfloat16).t()
    elif what == "x_strided":
        X = torch.zeros(12, 10, dtype=torch.bfloat16).t()
    elif what == "x_overlap":
        X = torch.zeros(1, 12, dtype=torch.bfloat16).expand(10, 12)
    elif what == "x_vector":
        X = X[0]
    elif what == "bias":
        kw["bias"] = torch.zeros(21, dtype=torch.bfloat16)
    elif what == "bias_dtype":
        kw["bias"] = torch.zeros(20)
    elif what == "residual":
        kw["residual"] = torch.zeros(10, 21, dtype=torch.bfloat16)
    elif what == "residual_dtype":
        kw["residual"] = torch.zeros(10, 20)
    elif what == "y":
        kw["out"] = {"Y": torch.zeros(11, 20, dtype=torch.bfloat16)}
    elif what == "z":
        kw["out"] = {"Z": torch.zeros(10, 24, dtype=torch.bfloat16)[:, :20]}
    elif what == "rng_dtype":
        kw["rng"] = torch.zeros(2)
    elif what == "rng_shape":
        kw["rng"] = torch.zeros(3, dtype=torch.int64)
    elif what == "p":
        kw["dropout"] = 1.5
    elif what == "call":
        kw["call"] = -1
    with pytest.raises(ValueError, match=text):
        mhffn.linear_forward(X, W, **kw)


@pytest.mark.parametrize("what,error,text", [
    ("dy", ValueError, "dY must be"), ("z", ValueError, "Z must have shape"), ("want", KeyError, "dR"),
    ("dx_stride", ValueError, "row stride"), ("dw", ValueError, "dW must be contiguous"),
    ("dbias", ValueError, "dbias has dtype"), ("device", ValueError, "X is on cpu")])
def test_linear_backward_says_what_is_wrong(what, error, text):
    X, W = _args()
    dY, kw = torch.zeros(10, 20, dtype=torch.bfloat16), {}
    if what == "dy":
        dY = torch.zeros(10, 12, dtype=torch.bfloat16)
    elif what == "z":
        kw["Z"] = torch.zeros(9, 20, dtype=torch.bfloat16)
    elif what == "want":
        kw["want"] = ("dX", "dR")
    elif what == "dx_stride":
        kw["out"] = {"dX": torch.zeros(10, 16, dtype=torch.bfloat16)[:, :12]}
    elif what == "dw":
        kw["out"] = {"dW": torch.zeros(20, 12, dtype=torch.bfloat16).t()}
    elif what == "dbias":
        kw["out"] = {"dbias": torch.zeros(20)}
    with pytest.raises(error, match=text):
        mhffn.linear_backward(X, W, dY, **kw)


@pytest.mark.parametrize("kw,text", [
    (dict(residual=torch.zeros(10, 13)), "residual must be"), (dict(out=torch.zeros(10, 12, dtype=torch.int32)), "out has dtype"),
    (dict(rng=torch.zeros(2, dtype=torch.int32)), "rng has dtype"), (dict(p=-0.5), "dropout must be"), ({}, "X is on cpu")])
def test_dropout_says_what_is_wrong(kw, text):
    kw = {"p": 0.5, "rng": torch.zeros(2, dtype=torch.int64), **kw}
    with pytest.raises(ValueError, match=text):
        mhffn.dropout(torch.zeros(10, 12), **kw)
    with pytest.raises(TypeError):
        mhffn.dropout(torch.zeros(10, 12, dtype=torch.float16), 0.5, kw["rng"])


def test_the_module_with_a_residual_says_what_is_wrong():
    X, P = torch.zeros(8, 256, dtype=torch.bfloat16), torch.zeros(256, 256, dtype=torch.bfloat16)
    W = [torch.zeros(2, 3, 64, 128, dtype=torch.bfloat16) for _ in range(3)]
    Wr = torch.zeros(2, 128, 3, dtype=torch.bfloat16)
    for kw, text in ((dict(residual=X[:, :128]), "residual must be"), (dict(dropout=2.0), "dropout must be"),
                     (dict(residual=X, rng=torch.zeros(2)), "rng has dtype"), (dict(residual=X), "X is on cpu")):
        with pytest.raises(ValueError, match=text):
            mhffn.module_forward(X, P, *W, Wr, P, **kw)
    with pytest.raises(ValueError, match="X is on cpu"):
        mhffn.module_backward(X, P, *W, Wr, P, X, X, X, dropout=0.5, rng=torch.zeros(2, dtype=torch.int64))
