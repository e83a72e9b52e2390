"""How far float32 sums of random terms may be from the exact ones: narrow enough to see a part of dY left out, or products that are cut
before they are added, which bounds that add up every rounding's worst are not."""
import numpy as np

from f8_reference import HALF_STEP, LEAST


def sum_room(rss, mags, additions, exact, dtype):
    """`additions` additions in float32, each off by at most half a step (2^-24 of its result), are a random walk: results of such sums are about
    `rss`, the root of the terms' sum of squares, or less on the way, errors are spread evenly over a step, so that the walk's standard
    deviation is at most 2^-24 rss sqrt(additions / 3); six of them, sqrt(12) < 3.5 times rss sqrt(additions).  Few additions are not a walk: two roundings of the
    sum of magnitudes beside it.  Then the result's own rounding."""
    lost = 2.0 ** -24 * (3.5 * np.sqrt(additions) * rss + 2 * mags)
    return lost + (np.abs(exact) + lost) * HALF_STEP[dtype] + LEAST[dtype]


def gradient_room(Y, X, parts, dtype):
    """Sums over rows of Y and X, of each part of Y."""
    return sum_room(np.sqrt((Y * Y).T @ (X * X)), np.abs(Y).T @ np.abs(X), parts * Y.shape[0] + 8, Y.T @ X, dtype)


def product_room(A, B, dtype):
    """Products of rows; for float32 results, whose terms are added as float32 adds."""
    return sum_room(np.sqrt((A * A) @ (B * B).T), np.abs(A) @ np.abs(B).T, A.shape[1] + 8, A @ B.T, dtype)


def cut_products(A, B):
    """What A B^T would be if, of every eight coordinates' products, each were cut at 2^-14 of the largest's power of two (as the 8-bit matrix
    instructions do)."""
    m, d = A.shape
    full = -(-d // 8) * 8
    A, B = (np.pad(V, ((0, 0), (0, full - d))).reshape(len(V), -1, 8) for V in (A, B))
    out = np.empty((m, len(B)))
    for i in range(m):
        p = A[i] * B                                              # [rows of B, groups, 8]
        top = np.abs(p).max(axis=2, keepdims=True)
        unit = np.exp2(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 14)
        out[i] = (np.trunc(p / unit) * unit).sum(axis=(1, 2))
    return out
