"""Inputs of the gradient of the weights that need every part of dY and whose results are exact in float32: the sum of a column's few live
rows, in quarters, has at most 24 bits.  On the device that is asked for, so that a test without a GPU can look at them."""
import torch

from f8_reference import TYPES

BITS = {"f32": 18, "f16": 11, "bf16": 8}            # of dY's numbers: parts of eight bits, three, two and one of them
LIVE = {"f32": 4, "f16": 64, "bf16": 256}           # rows of a column of the table that are not zero: 2^18 * 1.75 * (4 + 3) * 4 < 2^24

# (rows, columns of dY, coordinates), with what they take: (tile, whether the sum is cut) of float32, half precision, bfloat16
SHAPES = {
    (33, 260, 500): ("narrow", "narrow", "narrow"),
    (500, 99, 500): ("narrow parts", "narrow parts", "narrow parts"),
    (33, 501, 4100): ("small", "small", "small"),
    (1500, 100, 4100): ("small parts", "small parts", "narrow parts"),
    (4001, 100, 4101): ("small parts", "small parts", "small parts"),
    (33, 2051, 3900): ("wide", "square", "square"),
    (1500, 2304, 2050): ("square parts", "square parts", "small"),
    (4001, 2051, 2050): ("wide parts", "square parts", "square parts"),
    (12_000, 1030, 1000): ("wide parts", "wide parts", "small parts"),
    (100_000, 65, 960): ("wide parts", "wide parts", "wide parts"),
}


def numbers(dtype, m, n, d, device, live=None):
    """(dY [m, n], X [m, d]) in float64: whole numbers of all their bits, and quarters; rows times powers of two that cancel."""
    gen = torch.Generator(device=device).manual_seed(m + n + d)
    most = 2 ** BITS[dtype] - 1
    Y = torch.randint(-most, most + 1, (m, n), generator=gen, device=device).to(torch.float64)
    X = torch.zeros((m, d), dtype=torch.float64, device=device)
    k = min(LIVE[dtype] if live is None else live, m)
    rows = torch.randint(0, m, (k, d), generator=gen, device=device)
    signs = torch.randint(0, 2, (k, d), generator=gen, device=device) * 2 - 1
    X.scatter_(0, rows, signs * (4 + torch.randint(0, 4, (k, d), generator=gen, device=device)).to(torch.float64) / 4)
    size = torch.exp2(torch.randint(-3, 4, (m, 1), generator=gen, device=device).to(torch.float64))
    return Y / size, X * size


def cut_out(Y, dtype):
    """The same numbers in the type, as rows of a wider matrix of NaN that begin and end anywhere."""
    m, n = Y.shape
    wide = torch.full((m * (n + 5) + 3,), float("nan"), dtype=TYPES[dtype], device=Y.device)
    out = wide[3:].view(m, n + 5)[:, :n]
    out.copy_(Y)
    return out


def upper_parts(Y, dtype, parts):
    """What is left of dY if only its first parts count, each the upper eight bits of what is left."""
    left, kept = Y.to(torch.float32), torch.zeros_like(Y)
    for _ in range(parts):
        part = (left.view(torch.int32) & -65536).view(torch.float32)
        kept += part.to(torch.float64)
        left = left - part
    return kept


COUNT = {"f32": 3, "f16": 2, "bf16": 1}


def special(dtype, m, n, d, device):
    """The same with infinities and NaN: (dY, X as a table is to hold it, (row, block) of a scale that stands for NaN, the exact result).  Rows of
    their own hold them, without zeros on the other side unless a zero is meant."""
    Y, X = numbers(dtype, m, n, d, device)
    in_y, in_x, nan_scale = m // 3, m // 2, m - 1
    gen = torch.Generator(device=device).manual_seed(7)
    X[in_y] = torch.randint(0, 2, (d,), generator=gen, device=device).to(torch.float64) * 2 - 1
    Y[in_y, n - 1], Y[in_y, 0] = float("inf"), float("nan")
    Y[in_x, ::3], Y[in_x, 1::5] = 2.0, 0.0                     # (later parts that are zero, and zeros)
    Y[in_x, 2::7] *= -1
    X[in_x] = 0.0
    X[in_x, d - 1], X[in_x, d - 2], X[in_x, 3] = float("inf"), float("nan"), -float("inf")
    X[nan_scale] = 0.0
    held = X.clone()
    held[nan_scale, 128:256] = float("nan")
    rest = torch.ones((m, 1), dtype=torch.float64, device=device)
    rest[[in_y, in_x, nan_scale]] = 0.0
    want = torch.where(rest == 0, 0.0, Y).T.contiguous() @ torch.where(rest == 0, 0.0, X)
    for t in (in_y, in_x, nan_scale):
        want = want + Y[t][:, None] * held[t][None, :]
    return Y, X, (nan_scale, 1), want
