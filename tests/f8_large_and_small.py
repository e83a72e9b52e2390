"""Rows whose products are small whole numbers, but for one large one in each of up to 64 blocks: sums that float32 holds exactly, of which the 8-bit
matrix instructions would cut the small ones that they add together with a large one."""
import numpy as np


def numbers(m, n, d):
    """(A [m, d], B [n, d]): 1 and 2 with signs, 448 at the same places of both, blocks times powers of two that cancel.  Sums are
    below 4 * 65536 + 64 * 448^2 < 2^24."""
    rng = np.random.default_rng([9, m, n, d])
    A, B = (rng.integers(1, 3, (k, d)) * (rng.integers(0, 2, (k, d)) * 2.0 - 1.0) for k in (m, n))
    blocks = -(-d // 128)
    large = rng.permutation(blocks)[:64]
    at = np.minimum(large * 128 + rng.integers(0, 128, len(large)), d - 1)
    A[:, at], B[:, at] = 448.0, 448.0 * (rng.integers(0, 2, (n, 1)) * 2 - 1)
    power = np.exp2(rng.integers(-6, 7, blocks)).repeat(128)[:d]
    return A * power, B / power
