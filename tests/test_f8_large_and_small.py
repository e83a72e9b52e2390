"""The numbers that tests of exact float32 products take, without a GPU: their sums are exact in float32, and products that are cut before they
are added do not give them."""
import numpy as np
import pytest

import f8_large_and_small
import f8_reference as ref
import f8_rooms


@pytest.mark.parametrize("m,n,d", [(3, 7, 64), (2, 17, 129), (33, 40, 1100), (4, 6, 5000), (2, 3, 16384), (2, 3, 65536)])
def test_sums_are_exact_and_need_every_product(m, n, d):
    A, B = f8_large_and_small.numbers(m, n, d)
    for form in ("e4m3", "e5m2"):
        for V in (A, B):
            assert np.array_equal(ref.held(*ref.quantise(V, form), d, form), V)
    want = A @ B.T
    assert np.array_equal(want.astype(np.float32), want) and np.abs(A) .max() > 0 and (np.abs(A) @ np.abs(B).T).max() < 2 ** 24
    assert (f8_rooms.cut_products(A, B) != want).mean() > 0.9
