"""The operators around the fused path: a linear layer with bias, activation, dropout and residual
in its epilogue, its backward, and dropout by itself.  What a model that holds the module asks of
them, from one decoded token to a training batch.

  op         one pass
  forward    Y = R + D(act(X W + b)), and the pre-activation Z = X W + b where a training step keeps it
  backward   dX, dW and db of the same layer from X, W, Z and dY
  dropout    Y = R + D(X), or D(X): forward and backward of a dropout that stands alone

A case names the rows, the widths, the storage type, the activation, the dropout probability and
which of bias, residual and Z there are.  D keeps an element or sets it to zero.  Its random numbers are
those of Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): key = the seed, counter = (block, offset + call),
a block being eight neighbouring columns of a row, one 16-bit half of the four words each.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTIVATIONS = ("none", "relu", "silu", "gelu")
CALL = 3          # which of a step's dropouts this one is


def _case(op, rows, d_in, d_out, dtype="bf16", act="none", p=0.0, bias=False, residual=False, keep_z=False, name=None):
    c = {"op": op, "rows": rows, "d_in": d_in, "d_out": d_out, "dtype": dtype, "act": act, "p": p, "bias": bias,
         "residual": residual, "keep_z": keep_z}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # The output projection of one decoded token at the 1.3B shape, onto the residual stream.
        _case("forward", 1, 2048, 2048, bias=True, residual=True, name="fwd_decode_1"),
        # A decoding batch through the first layer of a dense FFN of the 1.3B shape.
        _case("forward", 64, 2048, 5632, act="silu", bias=True, name="fwd_decode_64"),
        # A prompt of ragged length through the first layer of a dense FFN of the 370M shape.
        _case("forward", 1000, 1024, 2816, act="gelu", bias=True, name="fwd_prefill_1000"),
        # Widths that nothing divides (a classifier head, an adapter), in training.
        _case("forward", 777, 1001, 515, act="relu", p=0.1, bias=True, residual=True, name="fwd_odd_777"),
        # Training at the 1.3B shape: the output projection with its residual branch ...
        _case("forward", 16384, 2048, 2048, p=0.1, bias=True, residual=True, name="fwd_project_16384"),
        # ... and the first layer of a dense FFN, which keeps Z for its backward.
        _case("forward", 16384, 2048, 5632, act="gelu", bias=True, keep_z=True, name="fwd_up_16384"),
        # Full precision at the 128M shape, a ragged number of tokens.
        _case("forward", 2000, 768, 2048, dtype="f32", act="silu", bias=True, name="fwd_f32_2000"),
        # Backward: a projection on a short batch, the first layer of the dense FFN, odd widths in fp32.
        _case("backward", 1024, 1024, 1024, p=0.1, bias=True, name="bwd_project_1024"),
        _case("backward", 16384, 2048, 5632, act="gelu", bias=True, name="bwd_up_16384"),
        _case("backward", 1500, 515, 1001, dtype="f32", act="silu", p=0.1, bias=True, name="bwd_f32_odd"),
        # Dropout alone: on the residual stream of a training batch, and the backward of a short fp32 one.
        _case("dropout", 16384, 2048, 2048, p=0.1, residual=True, name="dropout_16384"),
        _case("dropout", 333, 1001, 1001, dtype="f32", p=0.25, name="dropout_odd_333"),
    ]


def _cost(c):
    """Work of a case on one scale: flops at the type's matrix rate (fp32: one sixteenth of bf16's),
    or the bytes' time."""
    w = work(c)
    return max(w["flops"] * (16 if c["dtype"] == "f32" else 1), w["bytes"] * 300)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    """Half of the widths are a model's, multiples of 64; the others are any number."""
    return 64 * _log_int(rng, 2, 128) if rng.random() < 0.5 else _log_int(rng, 33, 4099)


def _draw_once(rng):
    op = rng.choice(("forward", "forward", "forward", "backward", "backward", "dropout"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "dropout":
        width = _width(rng)
        return _case(op, _log_int(rng, 1, 32768), width, width, dtype, p=rng.choice((0.05, 0.1, 0.25, 0.5)),
                     residual=rng.random() < 0.5)
    act = rng.choice(ACTIVATIONS)
    rows = _log_int(rng, 1 if op == "forward" else 64, 16384)
    p = rng.choice((0.0, 0.1, 0.25)) if rows >= 64 else 0.0
    return _case(op, rows, _width(rng), _width(rng), dtype, act=act, p=p, bias=rng.random() < 0.75,
                 residual=op == "forward" and rng.random() < 0.5,
                 keep_z=op == "forward" and act != "none" and rows >= 64 and rng.random() < 0.5)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        if _cost(c) <= most:
            return c


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    M, K, N = case["rows"], case["d_in"], case["d_out"]
    if case["op"] == "dropout":
        return {"bytes": es * M * N * (3 if case["residual"] else 2), "flops": 2 * M * N}
    if case["op"] == "forward":
        outs = 1 + int(case["residual"]) + int(case["keep_z"])
        return {"bytes": es * (M * K + K * N + int(case["bias"]) * N + outs * M * N), "flops": 2 * M * N * K}
    ins = 1 + int(case["act"] != "none")
    return {"bytes": es * (2 * M * K + 2 * K * N + N + ins * M * N), "flops": 4 * M * N * K}


def prepare(case, seed):
    """The tensors of one pass: activations and gradients of unit scale, weights of scale
    1 / sqrt(d_in), a small bias, and the generator's state."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    M, K, N = case["rows"], case["d_in"], case["d_out"]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    s = {"case": case, "X": normal(M, K), "rng": torch.tensor([seed * 7919 + 17, seed % 1000], device="cuda")}
    s["residual"] = normal(M, N) if case["residual"] else None
    if case["op"] == "dropout":
        return s
    s["W"] = normal(K, N, scale=K ** -0.5)
    s["bias"] = normal(N, scale=0.1) if case["bias"] else None
    if case["op"] == "backward":
        s["Z"] = normal(M, N) if case["act"] != "none" else None
        s["dY"] = normal(M, N)
    return s


# ---- plain form -------------------------------------------------------------------------------
def _keep(rng, rows, cols, threshold):
    """Which elements of a [rows, cols] array stay."""
    low, blocks = 0xFFFFFFFF, (cols + 7) // 8
    step = rng[1] + CALL
    block = torch.arange(rows * blocks, device=rng.device)
    a, b, c, d = block & low, block >> 32, (step & low).expand_as(block), ((step >> 32) & low).expand_as(block)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low

    def product(x, m):       # the two halves of a product of 64 bits
        return (((x * (m & 0xFFFF)) >> 16) + x * (m >> 16)) >> 16, (x * m) & low

    for _ in range(10):      # the generator's ten rounds
        hi0, lo0 = product(a, 0xD2511F53)
        hi1, lo1 = product(c, 0xCD9E8D57)
        a, b, c, d = hi1 ^ b ^ k0, lo1, hi0 ^ d ^ k1, lo0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((a, b, c, d), -1)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1)
    return halves.view(rows, blocks * 8)[:, :cols] >= threshold


def _dropout(v, rng, p):
    threshold = round(p * 65536)
    if threshold == 0:
        return v
    return torch.where(_keep(rng, *v.shape, threshold), v * (65536.0 / (65536 - threshold)), 0.0)


def _activation(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _slope(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, 1.0)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5


def _plain(s):
    c, dtype = s["case"], s["X"].dtype
    x = s["X"].float()
    if c["op"] == "dropout":
        y = _dropout(x, s["rng"], c["p"])
        return (y if s["residual"] is None else y + s["residual"].float()).to(dtype)
    w = s["W"].float()
    if c["op"] == "forward":
        z = x @ w
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _dropout(_activation(z, c["act"]), s["rng"], c["p"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(dtype), z.to(dtype)) if c["keep_z"] else y.to(dtype)
    dz = _dropout(s["dY"].float(), s["rng"], c["p"])
    if c["act"] != "none":
        dz = dz * _slope(s["Z"].float(), c["act"])
    return {"dX": (dz @ w.T).to(dtype), "dW": (x.T @ dz).to(dtype), "dbias": dz.sum(0).to(dtype)}


# ---- the framework's operators ----------------------------------------------------------------
def _framework(s):
    from paper_2512_06989_amd import mhffn
    c = s["case"]
    act = {"none": mhffn.ACT_NONE, "relu": mhffn.ACT_RELU, "silu": mhffn.ACT_SILU, "gelu": mhffn.ACT_GELU}[c["act"]]
    if c["op"] == "dropout":
        return mhffn.dropout(s["X"], c["p"], s["rng"], call=CALL, residual=s["residual"])
    if c["op"] == "forward":
        return mhffn.linear_forward(s["X"], s["W"], s["bias"], s["residual"], activation=act, dropout=c["p"],
                                    rng=s["rng"], call=CALL, save=c["keep_z"])
    return mhffn.linear_backward(s["X"], s["W"], s["dY"], s["Z"], activation=act, dropout=c["p"], rng=s["rng"],
                                 call=CALL)


def run(state):
    return _framework(state) if own else _plain(state)


# ---- in 64 bits, from the definition ----------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    M, N, f64 = case["rows"], case["d_out"], torch.float64
    threshold = int(np.rint(np.float32(case["p"]) * np.float32(65536)))
    scaled = torch.ones(M, N, dtype=f64, device="cuda")
    if threshold:
        u32, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
        seed_word, step = (np.uint64(int(v)) for v in s["rng"].cpu() + torch.tensor([0, CALL]))
        per_row = -(-N // 8)
        ctr = [np.arange(M * per_row, dtype=np.uint64), None, np.uint64(step) & u32, np.uint64(step) >> shift]
        ctr[0], ctr[1] = ctr[0] & u32, ctr[0] >> shift
        key = [int(seed_word & u32), int(seed_word >> shift)]
        for _ in range(10):
            p, q = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            ctr = [(q >> shift) ^ ctr[1] ^ np.uint64(key[0]), q & u32, (p >> shift) ^ ctr[3] ^ np.uint64(key[1]), p & u32]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        bits = np.stack([w.astype("<u4") for w in ctr], axis=1).view("<u2").reshape(M, per_row * 8)[:, :N]
        scaled = torch.from_numpy(bits >= threshold).cuda() * (65536.0 / (65536 - threshold))
    x = s["X"].to(f64)
    r = 0.0 if s["residual"] is None else s["residual"].to(f64)
    if case["op"] == "dropout":
        return x * scaled + r

    def gate(t):     # act(t) / t
        return {"none": lambda: torch.ones_like(t), "relu": lambda: (t > 0).to(f64), "silu": lambda: torch.sigmoid(t),
                "gelu": lambda: 0.5 * torch.special.erfc(-t / math.sqrt(2))}[case["act"]]()

    def gate_slope(t):   # t times the derivative of act(t) / t
        if case["act"] == "silu":
            return t * torch.sigmoid(t) * torch.sigmoid(-t)
        return t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi) if case["act"] == "gelu" else torch.zeros_like(t)

    w = s["W"].to(f64)
    if case["op"] == "forward":
        z = torch.mm(x, w)
        if s["bias"] is not None:
            z += s["bias"].to(f64)
        y = z * gate(z) * scaled + r
        return (y, z) if case["keep_z"] else y
    dz = s["dY"].to(f64) * scaled
    if s["Z"] is not None:
        z = s["Z"].to(f64)
        dz = dz * (gate(z) + gate_slope(z))
    return {"dX": torch.mm(dz, w.t().contiguous()), "dW": torch.mm(x.t().contiguous(), dz), "dbias": dz.sum(0)}
