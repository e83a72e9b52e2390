"""A plain statement, in 64 bits, of the 8-bit format with a scale per block of 128 and of the operators on it."""
import numpy as np
import torch

FORMS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}     # half of the smallest number


def code_values(form):
    """Values of the 256 codes."""
    bits, bias = (3, 7) if form == "e4m3" else (2, 15)
    out = np.empty(256)
    for c in range(256):
        e, man = (c & 127) >> bits, c & (2 ** bits - 1)
        v = man * 2.0 ** (1 - bias - bits) if e == 0 else (2 ** bits + man) * 2.0 ** (e - bias - bits)
        if form == "e4m3" and c & 127 == 127:
            v = np.nan
        if form == "e5m2" and c & 127 >= 124:
            v = np.inf if c & 127 == 124 else np.nan
        out[c] = -v if c & 128 else v
    return out


def exponents(top, form):
    """Smallest e from -127 on with top <= 1.75 * 2^(8 or 15) * 2^e."""
    most = 448.0 if form == "e4m3" else 57344.0
    e = np.full(top.shape, -127.0)
    live = top > 0
    e[live] = np.maximum(np.ceil(np.log2(top[live] / most)) - 2, -127)
    for _ in range(4):
        e = np.where(top > most * 2.0 ** e, e + 1, e)
    return e


def codes_of(x, form):
    """Codes (uint8) of numbers within the format's range: nearest, ties to the even code."""
    value = code_values(form)[:127 if form == "e4m3" else 124]
    mag = np.abs(x)
    hi = np.clip(np.searchsorted(value, np.where(np.isfinite(mag), mag, 0.0)), 0, len(value) - 1)
    lo = np.maximum(hi - 1, 0)
    with np.errstate(invalid="ignore"):
        up, down = value[hi] - mag, mag - value[lo]
        c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    c = np.where(np.isfinite(mag), c, 127 if form == "e4m3" else np.where(np.isnan(mag), 127, 124)).astype(np.uint8)
    return c | (np.signbit(x).astype(np.uint8) << 7)


def quantise(x, form, tall=1):
    """(codes [n, 128 nb], scales [n, sp]) of float64 rows, a scale for each `tall` x 128."""
    n, d = x.shape
    nb = (d + 127) // 128
    full = np.zeros((n, nb * 128))
    full[:, :d] = x
    blocks = full.reshape(n, nb, 128)
    top = np.where(np.isfinite(blocks), np.abs(blocks), 0.0).max(axis=2)
    if tall > 1:
        for r in range(0, n, tall):
            top[r:r + tall] = top[r:r + tall].max(axis=0, keepdims=True)
    e = exponents(top, form)
    scales = np.zeros((n, (nb + 3) // 4 * 4), np.uint8)
    scales[:, :nb] = (e + 127).astype(np.uint8)
    return codes_of(blocks / (2.0 ** e)[:, :, None], form).reshape(n, nb * 128), scales


def held(codes, scales, d, form):
    n, nb = codes.shape[0], (d + 127) // 128
    p = 2.0 ** (scales[:, :nb].astype(np.float64) - 127)
    p[scales[:, :nb] == 255] = np.nan
    return (code_values(form)[codes].reshape(n, nb, 128) * p[:, :, None]).reshape(n, nb * 128)[:, :d]


def host(t):
    t = t.detach()
    if t.dtype in (torch.float8_e4m3fn, torch.float8_e5m2):
        return t.view(torch.uint8).cpu().numpy()
    return t.cpu().to(torch.float64).numpy() if t.dtype.is_floating_point else t.cpu().numpy()


def form_of(table):
    return "e4m3" if table.codes.dtype == torch.float8_e4m3fn else "e5m2"


def held_by(table):
    return held(host(table.codes), host(table.scales), table.d, form_of(table))


def product_room(A, B, dtype):
    """How far a product may be from the exact one: sums of d terms in float32, each addition off by at most a step
    (2^-23) of the sum of magnitudes, and a rounding to the type; for 16 bits, what the 8-bit instructions cut off (2^-11 of
    the magnitudes: seven of eight products, each by less than 2^-14 of the largest)."""
    mags = np.abs(A) @ np.abs(B).T
    lost = (A.shape[1] + 8) * 2.0 ** -23 * mags
    if dtype != torch.float32:
        lost = lost + 2.0 ** -11 * mags
    exact = np.abs(A @ B.T)
    return lost + (exact + lost) * HALF_STEP[dtype] + LEAST[dtype]


def gradient_room(Y, X, dtype):
    """Likewise for sums over the rows, up to three parts each."""
    mags = np.abs(Y).T @ np.abs(X)
    lost = (3 * Y.shape[0] + 8) * 2.0 ** -23 * mags
    return lost + (np.abs(Y.T @ X) + lost) * HALF_STEP[dtype] + LEAST[dtype]
