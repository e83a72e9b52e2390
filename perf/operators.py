"""Timed cases of the operators on vectors held in microscaled 4-bit floating point (MXFP4).

A row of d coordinates is held as blocks of 32: a code of 4 bits per coordinate (E2M1: sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6) and a byte per block, the power of two (E8M0, bias 127) that its codes are
multiplied by.  The power is that of the block's largest magnitude, two less, so that the largest
magnitude is between 4 and 8 of it; codes are rounded to nearest, ties to the even code, and end at 6.
A table is `codes` [n, 16 * blocks] (low nibble first), `scales` [n, blocks rounded up to 4] and `norms`
[n], the squared lengths of the rows as they are held.

A case is a dict:
  op      "quantise"  rows -> table, and the rows as the table holds them read back, all of them
          "rows"      rows of a table by id, times a factor; an id below zero names an empty slot, a row of zeros
          "product"   A B^T of two tables
          "nearest"   float32 queries -> table -> the k nearest rows of another table by squared distance,
                      in the order (distance, id)
  data    distribution of the vectors: "gauss", "u8grid", "unit", "mixed" as in the package's synthetic
          workloads, or "layer": activations with a few large channels against weights
  n, d    rows and coordinates of the table;  m rows of A, ids or queries;  k results
  dtype   "f32", "f16" or "bf16": type of the rows that are quantised, or of the output
  pad     (quantise) coordinates between the end of a row and the next one
  own_rows (nearest) the queries are the table's first m vectors, and no vector is its own neighbour
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # an online batch of 64 query vectors as an encoder hands them over: latency
        dict(name="quantise_64_d128_bf16", op="quantise", data="unit", n=64, d=128, dtype="bf16", pad=0),
        # a whole descriptor set of the headline configuration, once when the index is made
        dict(name="quantise_1m_d128_f32", op="quantise", data="u8grid", n=1_000_000, d=128, dtype="f32", pad=0),
        # rows that end inside a block, cut out of a wider half-precision matrix
        dict(name="quantise_200003_d50_f16", op="quantise", data="gauss", n=200_003, d=50, dtype="f16", pad=7),
        # the candidates of 64 queries, 10 each, read back for a second look at them
        dict(name="rows_640_of_200003_d50_f32", op="rows", data="gauss", n=200_003, d=50, m=640, dtype="f32"),
        # the neighbours of every point of the middle configuration (degree 20), for a step that works on them
        dict(name="rows_2m_of_100k_d128_bf16", op="rows", data="u8grid", n=100_000, d=128, m=2_000_000, dtype="bf16"),
        # one query scored against a million rows
        dict(name="product_1_x_1m_d128_f32", op="product", data="u8grid", m=1, n=1_000_000, d=128, dtype="f32"),
        # a batch of queries scored against a shard of long vectors
        dict(name="product_4096_x_65536_d960_bf16", op="product", data="unit", m=4096, n=65_536, d=960, dtype="bf16"),
        # a large square layer, where the matrix units are the limit
        dict(name="product_8192_x_8192_d8192_bf16", op="product", data="layer", m=8192, n=8192, d=8192, dtype="bf16"),
        # one online query, exhaustively
        dict(name="nearest_1_of_1m_d128_k10", op="nearest", data="u8grid", m=1, n=1_000_000, d=128, k=10,
             own_rows=False),
        # the start of a graph over a set that is a multiple of nothing: every vector's neighbours among the others
        dict(name="nearest_graph_20003_d50_k15", op="nearest", data="gauss", m=20_003, n=20_003, d=50, k=15,
             own_rows=True),
        # a batch against a million long vectors (the largest vectors of the configurations)
        dict(name="nearest_1000_of_1m_d960_k10", op="nearest", data="unit", m=1000, n=1_000_000, d=960, k=10,
             own_rows=False),
        # the headline set and the 10 000 rows that recall is measured on: the truth a graph is compared with
        dict(name="nearest_10k_of_1m_d128_k10", op="nearest", data="u8grid", m=10_000, n=1_000_000, d=128, k=10,
             own_rows=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges that the listed ones stand for: tables of up to a million rows, from one row and one
    coordinate on, none with more work than the largest listed case of its operator."""
    op = rng.choice(["quantise", "rows", "product", "nearest"])
    data = rng.choice(["gauss", "u8grid", "unit", "mixed"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "quantise":
        d = _log_int(rng, 1, 1024)
        n = _log_int(rng, 1, min(1_000_000, 128_000_000 // d))
        return dict(op=op, data=data, n=n, d=d, dtype=dtype, pad=rng.choice([0, 0, 1, 8, 31]))
    if op == "rows":
        d = _log_int(rng, 8, 1024)
        n = _log_int(rng, 1, min(1_000_000, 128_000_000 // d))
        m = _log_int(rng, 1, min(2_000_000, 128_000_000 // d))
        return dict(op=op, data=data, n=n, d=d, m=m, dtype=dtype)
    if op == "product":
        if rng.random() < 0.3:
            data = "layer"
        d = _log_int(rng, 16, 8192)
        m = _log_int(rng, 1, 8192)
        n = _log_int(rng, 16, min(1_000_000, 268_000_000 // m, 536_000_000 // d,
                                  max(16, 549_000_000_000 // (m * d))))
        return dict(op=op, data=data, m=m, n=n, d=d, dtype=dtype)
    d = _log_int(rng, 8, 1024)
    k = _log_int(rng, 1, 100)
    n = _log_int(rng, 1000, 1_000_000)
    m = _log_int(rng, 1, min(10_000, int(1.28e12 / n / d)))
    own_rows = rng.random() < 0.3
    if own_rows:
        m = min(m, n)
    return dict(op=op, data=data, m=m, n=n, d=d, k=k, own_rows=own_rows)


# ---- inputs --------------------------------------------------------------------------------------------------------------


def _vectors(data, n, d, gen, centres=None):
    """(n vectors of a mixture, its centres), drawn on the GPU; one component per thousand rows."""
    lo, hi, sigma = {"gauss": (-10.0, 10.0, 1.0), "u8grid": (0.0, 128.0, 16.0), "unit": (0.0, 1.0, 0.05),
                     "mixed": (-1.0, 1.0, 0.1)}[data]
    if centres is None:
        centres = lo + (hi - lo) * torch.rand((max(10, n // 1000), d), generator=gen, device="cuda")
    comp = torch.randint(0, centres.shape[0], (n,), generator=gen, device="cuda")
    X = torch.empty((n, d), dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=gen)
    for r in range(0, n, 1 << 18):
        X[r:r + (1 << 18)] += centres[comp[r:r + (1 << 18)]]
    if data == "u8grid":
        X.clamp_(0.0, 255.0).round_()
    elif data == "unit":
        X.clamp_(0.0, 1.0)
    elif data == "mixed":
        flat = torch.rand((n,), generator=gen, device="cuda") < 0.5
        X[flat] = torch.rand((int(flat.sum()), d), generator=gen, device="cuda") * 2.0 - 1.0
    return X, centres


def _pair_of_sets(case, gen):
    """Float32 rows of the table and of what meets it (queries, or the left factor)."""
    n, m, d = case["n"], case["m"], case["d"]
    if case["data"] == "layer":
        W = torch.empty((n, d), device="cuda").normal_(0.0, d ** -0.5, generator=gen)
        A = torch.empty((m, d), device="cuda").normal_(0.0, 1.0, generator=gen)
        A[:, torch.rand((d,), generator=gen, device="cuda") < 0.01] *= 10.0
        return W, A
    X, centres = _vectors(case["data"], n, d, gen)
    if case.get("own_rows"):
        return X, X[:m].contiguous()
    return X, _vectors(case["data"], m, d, gen, centres)[0]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "quantise":
        X, _ = _vectors(case["data"], case["n"], case["d"], gen)
        wide = torch.zeros((case["n"], case["d"] + case["pad"]), dtype=DTYPE[case["dtype"]], device="cuda")
        wide[:, :case["d"]] = X
        return dict(x=wide[:, :case["d"]])
    if case["op"] == "rows":
        X, _ = _vectors(case["data"], case["n"], case["d"], gen)
        ids = torch.randint(0, case["n"], (case["m"],), generator=gen, device="cuda", dtype=torch.int32)
        ids[torch.rand((case["m"],), generator=gen, device="cuda") < 0.01] = -1      # rows of a graph that are not full
        return dict(table=_quantise(X), ids=ids, factor=case["d"] ** -0.5)
    X, A = _pair_of_sets(case, gen)
    if case["op"] == "product":
        return dict(table=_quantise(X), a=_quantise(A))
    return dict(table=_quantise(X), queries=A)


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own:
        from paper_1609_07228_amd import efanna
        state["lib"] = efanna
        for key in ("table", "a"):
            if key in state:
                state[key] = efanna.MxTable(*state[key])
    return state


# ---- the plain forms -------------------------------------------------------------------------------------------------------


def _quantise(x):
    """(codes, scales, norms, d) of the rows of x, by comparisons in float32."""
    n, d = x.shape
    nb = (d + 31) // 32
    xb = torch.zeros((n, nb * 32), dtype=torch.float32, device=x.device)
    xb[:, :d] = x
    xb = xb.view(n, nb, 32)
    mag = xb.abs()
    top = mag.amax(dim=2)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127)
    mag = torch.ldexp(mag, -e[:, :, None])
    code = torch.zeros(mag.shape, dtype=torch.uint8, device=x.device)
    for border, above in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (mag >= border) if above else (mag > border)
    code += torch.signbit(xb).to(torch.uint8) * 8
    code = code.view(n, nb * 32)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    scales = torch.zeros((n, (nb + 3) // 4 * 4), dtype=torch.uint8, device=x.device)
    scales[:, :nb] = (e + 127).to(torch.uint8)
    held = _held(codes, scales, d)
    return codes, scales, (held * held).sum(dim=1), d


def _held(codes, scales, d):
    """Float32 rows that a table stands for."""
    value = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float32, device=codes.device)
    pair = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1)
    nb = (d + 31) // 32
    power = torch.ldexp(torch.ones((), device=codes.device), scales[:, :nb].to(torch.int32) - 127)
    return (value[pair.to(torch.int32)].view(-1, nb, 32) * power[:, :, None]).view(-1, nb * 32)[:, :d]


def _nearest(table, a, k, own_rows):
    """k largest q.x - |x|^2 / 2 of every query, equal ones by the lower id, as (ids, squared distances)."""
    X, Q = _held(table[0], table[1], table[3]), _held(a[0], a[1], a[3])
    n = X.shape[0]
    half = 0.5 * table[2]
    step = max(1, (1 << 27) // n)
    row = torch.arange(n, device=X.device)
    ids, dists = [], []
    for q0 in range(0, Q.shape[0], step):
        s = Q[q0:q0 + step] @ X.T - half
        order = (0.0 - s).view(torch.int32)
        order = (order ^ ((order >> 31) & 0x7FFFFFFF)).to(torch.int64)
        key = (order << 32) + row
        if own_rows:
            here = torch.arange(s.shape[0], device=X.device)
            key[here, here + q0] = torch.iinfo(torch.int64).max
        got = (key.topk(k, dim=1, largest=False, sorted=True).values & 0xFFFFFFFF)
        ids.append(got.to(torch.int32))
        dists.append((a[2][q0:q0 + step, None] - 2.0 * s.gather(1, got)).clamp(min=0.0))
    return torch.cat(ids), torch.cat(dists)


def _plain(state):
    case = state["case"]
    if case["op"] == "quantise":
        codes, scales, norms, d = _quantise(state["x"])
        return _held(codes, scales, d).to(DTYPE[case["dtype"]]), norms
    if case["op"] == "rows":
        codes, scales, _, d = state["table"]
        ids = state["ids"].to(torch.int64)
        at = ids.clamp(min=0)
        out = _held(codes[at], scales[at], d) * state["factor"]
        return torch.where(ids[:, None] < 0, 0.0, out).to(DTYPE[case["dtype"]])
    if case["op"] == "product":
        a, b = (_held(t[0], t[1], t[3]) for t in (state["a"], state["table"]))
        return (a @ b.T).to(DTYPE[case["dtype"]])
    return _nearest(state["table"], _quantise(state["queries"]), case["k"], case["own_rows"])


def run(state):
    if not own:
        return _plain(state)
    case, lib = state["case"], state["lib"]
    if case["op"] == "quantise":
        table = lib.efanna_mx_quantise(state["x"])
        return lib.efanna_mx_rows(table, dtype=DTYPE[case["dtype"]]), table.norms
    if case["op"] == "rows":
        return lib.efanna_mx_rows(state["table"], state["ids"], factor=state["factor"], dtype=DTYPE[case["dtype"]])
    if case["op"] == "product":
        return lib.efanna_mx_product(state["a"], state["table"], dtype=DTYPE[case["dtype"]])
    queries = lib.efanna_mx_quantise(state["queries"])
    return lib.efanna_mx_nearest(state["table"], queries, case["k"], first_self=0 if case["own_rows"] else -1)


def work(case):
    def table(n):
        nb = (case["d"] + 31) // 32
        return n * (16 * nb + (nb + 3) // 4 * 4)
    size = {"f32": 4, "f16": 2, "bf16": 2}
    n, d = case["n"], case["d"]
    if case["op"] == "quantise":        # rows in, table, norms and the rows read back out
        return dict(bytes=2 * n * d * size[case["dtype"]] + table(n) + 4 * n, flops=6 * n * d)
    m = case["m"]
    if case["op"] == "rows":            # a row that is named more than once need not come from memory again
        return dict(bytes=table(min(n, m)) + m * (4 + d * size[case["dtype"]]), flops=2 * m * d)
    if case["op"] == "product":
        return dict(bytes=table(n) + table(m) + m * n * size[case["dtype"]], flops=2 * m * n * d)
    return dict(bytes=table(n) + 4 * n + m * (4 * d + 8 * case["k"]), flops=2 * m * n * d)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------


def _exact_held(x):
    """What the format keeps of x, float64: the nearest multiple of the step that the magnitude's octave has."""
    x = x.to(torch.float64)
    n, d = x.shape
    out = torch.empty_like(x)
    for b in range(0, d, 32):
        block = x[:, b:b + 32]
        top = block.abs().amax(dim=1, keepdim=True)
        e = torch.where(top > 0, torch.frexp(top)[1].to(torch.float64) - 3.0, -127.0).clamp(min=-127.0)
        unit = torch.pow(torch.full_like(e, 2.0), e)
        a = block.abs() / unit
        step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
        out[:, b:b + 32] = torch.sign(block) * (torch.round(a / step) * step).clamp(max=6.0) * unit
    return out


def _exact_read(table):
    """Rows of a table, float64, coordinate by coordinate from sign, exponent and mantissa bits."""
    codes, scales, _, d = table
    out = torch.empty((codes.shape[0], d), dtype=torch.float64, device=codes.device)
    for j in range(d):
        c = ((codes[:, j // 2] >> (4 * (j % 2))) & 15).to(torch.int64)
        expo, man = (c >> 1) & 3, (c & 1).to(torch.float64)
        v = torch.where(expo == 0, 0.5 * man, (1.0 + 0.5 * man) * torch.pow(2.0, (expo - 1).to(torch.float64)))
        out[:, j] = torch.where(c >= 8, -v, v) * torch.pow(2.0, scales[:, j // 32].to(torch.float64) - 127.0)
    return out


def _exact_nearest(X, Q, k, own_rows):
    n = X.shape[0]
    xx, qq = (X * X).sum(dim=1), (Q * Q).sum(dim=1)
    ids = torch.empty((Q.shape[0], k), dtype=torch.int32, device=X.device)
    dists = torch.empty((Q.shape[0], k), dtype=torch.float64, device=X.device)
    step = max(1, (1 << 27) // n)
    for q0 in range(0, Q.shape[0], step):
        q1 = min(Q.shape[0], q0 + step)
        dist = (qq[q0:q1, None] + xx - 2.0 * (Q[q0:q1] @ X.T)).clamp(min=0.0)
        if own_rows:
            here = torch.arange(q1 - q0, device=X.device)
            dist[here, here + q0] = math.inf
        limit = dist.topk(k, dim=1, largest=False).values[:, -1:]
        at = (dist <= limit).nonzero()                 # (query, id), ascending; ties at the limit among them
        near = dist[at[:, 0], at[:, 1]]
        by = near.argsort(stable=True)
        by = by[at[by, 0].argsort(stable=True)]
        at, near = at[by], near[by]
        first = torch.searchsorted(at[:, 0].contiguous(), torch.arange(q1 - q0, device=X.device))
        take = first[:, None] + torch.arange(k, device=X.device)
        ids[q0:q1], dists[q0:q1] = at[take, 1].to(torch.int32), near[take]
    return ids, dists


def exact(case, seed):
    got = _inputs(case, seed)
    if case["op"] == "quantise":
        held = _exact_held(got["x"])
        return held, (held * held).sum(dim=1)
    if case["op"] == "rows":
        ids = got["ids"].to(torch.int64)
        out = _exact_read(got["table"])[ids.clamp(min=0)] * got["factor"]
        out[ids < 0] = 0.0
        return out
    if case["op"] == "product":
        return _exact_read(got["a"]) @ _exact_read(got["table"]).T
    return _exact_nearest(_exact_read(got["table"]), _exact_held(got["queries"]), case["k"], case["own_rows"])
