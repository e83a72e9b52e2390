"""Timed cases of the operators on matrices held in 8-bit floating point with a scale for each block of 128.

A row of d coordinates is held as blocks of 128, the last one filled up with zeros: a code of 8 bits per
coordinate and a byte per block, the power of two (E8M0, bias 127) that its codes are multiplied by.  Codes are
"e4m3" (three bits of mantissa, up to 448) or "e5m2" (two, up to 57344).  The power is the smallest, from 2^-127 on,
that leaves no magnitude of the block beyond the largest code; codes are rounded to nearest, ties to the even
code.  A table is `codes` [n, 128 * blocks] and `scales` [n, blocks rounded up to 4].

A linear layer y = x w^T is trained with them: its input is kept in 8 bits for the backward pass, its weight is
held both ways round, the products y and dx are products of two tables, and dw takes dy and the input as held.

A case is a dict:
  op      "checkpoint"  activations -> table, and all of them read back
          "weights"     a weight matrix -> its table and the table of its transpose, one scale for each tile of
                        128 x 128, and both read back
          "product"     A B^T of two tables
          "gradient"    dy^T X of a matrix and a table with as many rows
  data    distribution of the values: "layer" (a few large channels), "relu" (half of them zero), "u8grid"
          (descriptors: whole numbers up to 255), "weight", "gradient" (rows of very different size, some zero)
  n, d    rows and coordinates of the table; for "product" m rows of A; for "gradient" m rows of dy and of the
          table, n columns of dy
  fmt     format of the codes; for "product" a_fmt and fmt, those of A and of B
  dtype   "f32", "f16" or "bf16": type of what is quantised, of dy, or of the output of a product
  out     ("gradient") type of the output
  pad     ("checkpoint", "gradient") elements between the end of a row (of dy) and the next one
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
MANTISSA = {"e4m3": 3, "e5m2": 2}
TOP = {"e4m3": 8, "e5m2": 15}            # exponent of the largest code, 1.75 * 2^TOP
LOW = {"e4m3": -6, "e5m2": -14}          # exponent of the smallest code with all its mantissa


def listed():
    return [
        # the outputs of an encoder for an online batch: latency
        dict(name="checkpoint_64_d128_bf16", op="checkpoint", data="layer", n=64, d=128, fmt="e4m3", dtype="bf16", pad=0),
        # rows that end inside a block, cut out of a wider half-precision matrix
        dict(name="checkpoint_200003_d50_f16", op="checkpoint", data="relu", n=200_003, d=50, fmt="e4m3", dtype="f16", pad=7),
        # the input of a wide layer, for a whole batch of tokens
        dict(name="checkpoint_65536_d4096_bf16", op="checkpoint", data="layer", n=65_536, d=4096, fmt="e4m3", dtype="bf16",
             pad=0),
        # a projection of the largest vectors of the configurations to the size of the headline's, after a step
        dict(name="weights_128_d960_f32", op="weights", data="weight", n=128, d=960, fmt="e4m3", dtype="f32"),
        # a large square layer's float32 weights, after a step
        dict(name="weights_8192_d8192_f32", op="weights", data="weight", n=8192, d=8192, fmt="e4m3", dtype="f32"),
        # one query scored against a million rows
        dict(name="product_1_x_1m_d128_f32", op="product", data="u8grid", m=1, n=1_000_000, d=128, a_fmt="e4m3", fmt="e4m3",
             dtype="f32"),
        # one token each of sixteen sequences through a large square layer
        dict(name="product_16_x_8192_d8192_bf16", op="product", data="layer", m=16, n=8192, d=8192, a_fmt="e4m3", fmt="e4m3",
             dtype="bf16"),
        # gradients on their way back through a layer whose sizes are multiples of nothing
        dict(name="product_1003_x_5001_d960_f16", op="product", data="gradient", m=1003, n=5001, d=960, a_fmt="e5m2",
             fmt="e4m3", dtype="f16"),
        # a large square layer, where the matrix units are the limit
        dict(name="product_8192_x_8192_d8192_bf16", op="product", data="layer", m=8192, n=8192, d=8192, a_fmt="e4m3",
             fmt="e4m3", dtype="bf16"),
        # a small layer and few rows: latency
        dict(name="gradient_1000_n50_d300_f16", op="gradient", data="relu", m=1000, n=50, d=300, fmt="e4m3", dtype="f16",
             out="f32", pad=3),
        # the projection from the largest vectors, trained on the whole middle configuration at once: few outputs, a long sum
        dict(name="gradient_100k_n128_d960_f32", op="gradient", data="layer", m=100_000, n=128, d=960, fmt="e4m3", dtype="f32",
             out="f32", pad=0),
        # a wide layer and a batch of tokens, where the matrix units are the limit
        dict(name="gradient_16384_n4096_d4096_bf16", op="gradient", data="layer", m=16_384, n=4096, d=4096, fmt="e4m3",
             dtype="bf16", out="f32", pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """A case of the ranges that the listed ones stand for, from one row and one coordinate on, none with more work than
    the largest listed case of its operator."""
    op = rng.choice(["checkpoint", "weights", "product", "gradient"])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "checkpoint":
        d = _log_int(rng, 1, 8192)
        n = _log_int(rng, 1, min(1_000_000, 134_000_000 // max(d, 128)))
        return dict(op=op, data=rng.choice(["layer", "relu", "u8grid", "gradient"]), n=n, d=d, fmt=fmt, dtype=dtype,
                    pad=rng.choice([0, 0, 1, 8, 31]))
    if op == "weights":
        return dict(op=op, data="weight", n=_log_int(rng, 1, 8192), d=_log_int(rng, 1, 8192), fmt=fmt, dtype=dtype)
    if op == "product":
        d = _log_int(rng, 16, 16_384)
        wide = max(d, 128)
        m = _log_int(rng, 1, 8192)
        n = _log_int(rng, 16, min(1_000_000, 268_000_000 // wide, 67_000_000 // m, 549_000_000_000 // (m * wide)))
        return dict(op=op, data=rng.choice(["layer", "relu", "u8grid", "gradient"]), m=m, n=n, d=d,
                    a_fmt=rng.choice(["e4m3", "e4m3", "e5m2"]), fmt=fmt, dtype=dtype)
    n, d = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
    limit = {"f32": 91_000_000_000, "f16": 137_000_000_000, "bf16": 274_000_000_000}[dtype]
    wide = max(n, d, 128)
    m = _log_int(rng, 1, min(200_000, 134_000_000 // wide, limit // (max(n, 128) * max(d, 128))))
    return dict(op=op, data=rng.choice(["layer", "relu", "u8grid"]), m=m, n=n, d=d, fmt=fmt, dtype=dtype,
                out=rng.choice(["f32", "f32", "bf16", "f16"]), pad=rng.choice([0, 0, 1, 8]))


# ---- inputs --------------------------------------------------------------------------------------------------------------


def _values(data, n, d, gen):
    """Float32 [n, d], drawn on the GPU."""
    x = torch.empty((n, d), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen)
    if data == "weight":
        return x.mul_(d ** -0.5)
    if data == "u8grid":
        return x.mul_(40.0).add_(64.0).clamp_(0.0, 255.0).round_()
    if data == "gradient":
        size = torch.rand((n, 1), generator=gen, device="cuda")
        x.mul_(torch.exp2(-10.0 * size) * 0.01)
        x[size[:, 0] < 0.01] = 0.0                     # padding of a batch: no gradient
        return x
    x[:, torch.rand((d,), generator=gen, device="cuda") < 0.01] *= 10.0
    return x.clamp_(min=0.0) if data == "relu" else x


def _apart(x, dtype, pad):
    """The same matrix in another type, cut out of one whose rows are `pad` longer."""
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=DTYPE[dtype], device="cuda")
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, d, fmt = case["n"], case["d"], case["fmt"]
    if case["op"] == "checkpoint":
        return dict(x=_apart(_values(case["data"], n, d, gen), case["dtype"], case["pad"]))
    if case["op"] == "weights":
        return dict(w=_values("weight", n, d, gen).to(DTYPE[case["dtype"]]))
    if case["op"] == "product":
        b = _values("u8grid" if case["data"] == "u8grid" else "weight", n, d, gen)
        a = _values(case["data"], case["m"], d, gen)
        return dict(a=_quantise(a, case["a_fmt"]), b=_quantise(b, fmt))
    dy = _apart(_values("gradient", case["m"], n, gen), case["dtype"], case["pad"])
    return dict(dy=dy, x=_quantise(_values(case["data"], case["m"], d, gen), fmt))


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own:
        from paper_1609_07228_amd import efanna_f8
        state["lib"] = efanna_f8
        for key in ("a", "b", "x"):
            if isinstance(state.get(key), tuple):
                state[key] = efanna_f8.F8Table(*state[key])
    return state


# ---- the plain forms -------------------------------------------------------------------------------------------------------


def _power(top, fmt):
    """Exponent of the smallest power of two, 2^-127 at least, that brings magnitudes up to `top` within the codes."""
    part, e = torch.frexp(top)                          # top = part * 2^e, part from 1/2 on and below 1
    e = e - 1 - TOP[fmt] + (part > 0.875)
    return torch.where(top > 0, e, -127).clamp(min=-127)


def _round(x, fmt):
    """The nearest code's value, ties to the even code; |x| is not beyond the largest code."""
    step = (torch.frexp(x)[1] - 1).clamp(min=LOW[fmt]) - MANTISSA[fmt]
    return torch.ldexp(torch.round(torch.ldexp(x, -step)), step)


def _blocks(x):
    """Float32 [n, blocks, 128] of rows, filled up with zeros."""
    n, d = x.shape
    nb = (d + 127) // 128
    out = torch.zeros((n, nb * 128), dtype=torch.float32, device=x.device)
    out[:, :d] = x
    return out.view(n, nb, 128)


def _packed(blocks, e, d, fmt):
    """(codes, scales, d) of blocks whose exponents are e [n, blocks]."""
    n, nb, _ = blocks.shape
    codes = _round(torch.ldexp(blocks, -e[:, :, None]), fmt).view(n, nb * 128).to(CODE[fmt])
    scales = torch.zeros((n, (nb + 3) // 4 * 4), dtype=torch.uint8, device=blocks.device)
    scales[:, :nb] = (e + 127).to(torch.uint8)
    return codes, scales, d


def _quantise(x, fmt):
    blocks = _blocks(x)
    return _packed(blocks, _power(blocks.abs().amax(dim=2), fmt), x.shape[1], fmt)


def _quantise_tiles(w, fmt):
    """The table of w and that of its transpose, a power for each tile of 128 x 128."""
    n, d = w.shape
    high, across = (n + 127) // 128, (d + 127) // 128
    full = torch.zeros((high * 128, across * 128), dtype=torch.float32, device=w.device)
    full[:n, :d] = w
    e = _power(full.view(high, 128, across, 128).abs().amax(dim=(1, 3)), fmt)
    rows = _packed(full[:n].view(n, across, 128), e.repeat_interleave(128, dim=0)[:n], d, fmt)
    turned = full.T.contiguous()[:d]
    return rows, _packed(turned.view(d, high, 128), e.T.repeat_interleave(128, dim=0)[:d], n, fmt)


def _held(table):
    """Float32 rows that a table stands for."""
    codes, scales, d = table
    n, nb = codes.shape[0], (d + 127) // 128
    e = scales[:, :nb].to(torch.int32) - 127
    return torch.ldexp(codes.to(torch.float32).view(n, nb, 128), e[:, :, None]).view(n, nb * 128)[:, :d]


def _plain(state):
    case = state["case"]
    if case["op"] == "checkpoint":
        return _held(_quantise(state["x"], case["fmt"])).to(DTYPE[case["dtype"]])
    if case["op"] == "weights":
        return tuple(_held(t).to(DTYPE[case["dtype"]]) for t in _quantise_tiles(state["w"], case["fmt"]))
    if case["op"] == "product":
        return (_held(state["a"]) @ _held(state["b"]).T).to(DTYPE[case["dtype"]])
    return (state["dy"].to(torch.float32).T @ _held(state["x"])).to(DTYPE[case["out"]])


def run(state):
    if not own:
        return _plain(state)
    case, lib = state["case"], state["lib"]
    if case["op"] == "checkpoint":
        table = lib.efanna_f8_quantise(state["x"], CODE[case["fmt"]])
        return lib.efanna_f8_rows(table, dtype=DTYPE[case["dtype"]])
    if case["op"] == "weights":
        table, turned = lib.efanna_f8_weights(state["w"], CODE[case["fmt"]])
        return lib.efanna_f8_rows(table, dtype=DTYPE[case["dtype"]]), lib.efanna_f8_rows(turned, dtype=DTYPE[case["dtype"]])
    if case["op"] == "product":
        return lib.efanna_f8_product(state["a"], state["b"], dtype=DTYPE[case["dtype"]])
    return lib.efanna_f8_gradient(state["dy"], state["x"], dtype=DTYPE[case["out"]])


def work(case):
    def table(n, d):
        nb = (d + 127) // 128
        return n * (128 * nb + (nb + 3) // 4 * 4)
    size = {"f32": 4, "f16": 2, "bf16": 2}
    n, d = case["n"], case["d"]
    if case["op"] == "checkpoint":          # rows in, the table and the rows read back out
        return dict(bytes=2 * n * d * size[case["dtype"]] + table(n, d), flops=4 * n * d)
    if case["op"] == "weights":             # a matrix in, two tables and two matrices out
        return dict(bytes=3 * n * d * size[case["dtype"]] + table(n, d) + table(d, n), flops=5 * n * d)
    m = case["m"]
    if case["op"] == "product":
        return dict(bytes=table(m, d) + table(n, d) + m * n * size[case["dtype"]], flops=2 * m * n * d)
    return dict(bytes=m * n * size[case["dtype"]] + table(m, d) + n * d * size[case["out"]], flops=2 * m * n * d)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------


def _code_values(fmt):
    """Values of the codes without a sign, ascending, float64: infinities and NaN left out."""
    bits = MANTISSA[fmt]
    bias = 7 if fmt == "e4m3" else 15
    out = []
    for code in range(127 if fmt == "e4m3" else 124):
        expo, man = code >> bits, code & ((1 << bits) - 1)
        out.append(man * 2.0 ** (1 - bias - bits) if expo == 0 else (2 ** bits + man) * 2.0 ** (expo - bias - bits))
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _exact_held(x, fmt, tall):
    """What the format keeps of x, float64, with a scale for each `tall` x 128 of it."""
    x = x.to(torch.float64)
    grid = _code_values(fmt)
    out = torch.empty_like(x)
    for r in range(0, x.shape[0], 4096):                # (a multiple of `tall`)
        for c in range(0, x.shape[1], 128):
            part = x[r:r + 4096, c:c + 128]
            top = part.abs().amax(dim=1)
            if tall > 1:
                top = torch.cat([p.amax().expand(p.shape[0]) for p in top.split(tall)])
            e = torch.full_like(top, -127.0)
            live = top > 0
            e[live] = torch.floor(torch.log2(top[live] / grid[-1])) - 1.0
            for _ in range(3):                          # (the logarithm may be off next to a power of two)
                e = torch.where(live & (top > grid[-1] * torch.exp2(e)), e + 1.0, e)
            unit = torch.exp2(e.clamp(min=-127.0))[:, None]
            mag = part.abs() / unit
            hi = torch.searchsorted(grid, mag).clamp(max=len(grid) - 1)
            lo = (hi - 1).clamp(min=0)
            up, down = grid[hi] - mag, mag - grid[lo]
            take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
            out[r:r + 4096, c:c + 128] = torch.sign(part) * grid[take] * unit
    return out


def _exact_read(table):
    """Rows of a table, float64, from sign, exponent and mantissa bits."""
    codes, scales, d = table
    fmt = "e4m3" if codes.dtype == CODE["e4m3"] else "e5m2"
    value = torch.zeros((128,), dtype=torch.float64, device="cuda")
    known = _code_values(fmt)
    value[:len(known)] = known
    byte = codes.view(torch.uint8)
    out = torch.empty((codes.shape[0], d), dtype=torch.float64, device="cuda")
    for c in range(0, d, 128):
        b = byte[:, c:min(c + 128, d)].to(torch.int32)
        v = torch.where(b >= 128, -1.0, 1.0) * value[b & 127]
        out[:, c:c + 128] = v * torch.exp2(scales[:, c // 128].to(torch.float64) - 127.0)[:, None]
    return out


def exact(case, seed):
    got = _inputs(case, seed)
    if case["op"] == "checkpoint":
        return _exact_held(got["x"], case["fmt"], 1)
    if case["op"] == "weights":
        held = _exact_held(got["w"], case["fmt"], 128)
        return held, held.T.contiguous()
    if case["op"] == "product":
        return _exact_read(got["a"]) @ _exact_read(got["b"]).T
    return got["dy"].to(torch.float64).T @ _exact_read(got["x"])
