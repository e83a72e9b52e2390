"""The bounds that float32 sums are tested with, without a GPU: they let float32 sums pass, and results with a part of dY left out, or of
products that are cut before they are added, do not."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import f8_parts  # noqa: E402
import f8_reference as ref  # noqa: E402
import f8_rooms  # noqa: E402

GRADIENTS = [(15, 50, 300), (300, 260, 520), (777, 384, 512)]
PRODUCTS = [(33, 32, 128), (40, 100, 257), (100, 200, 300), (129, 257, 640), (20, 300, 5000)]


def held(rng, n, d):
    return ref.held(*ref.quantise(rng.standard_normal((n, d)), "e4m3"), d, "e4m3")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("m,n,d", GRADIENTS)
def test_a_gradient_with_one_part_fewer_is_out_of_the_room(dtype, m, n, d):
    rng = np.random.default_rng([m, n, d])
    dy = torch.as_tensor(rng.standard_normal((m, n))).to(ref.TYPES[dtype])
    Y, X = dy.to(torch.float64).numpy(), held(rng, m, d)
    room = f8_rooms.gradient_room(Y, X, f8_parts.COUNT[dtype], torch.float32)
    fewer = f8_parts.upper_parts(dy.to(torch.float64), dtype, f8_parts.COUNT[dtype] - 1).numpy()
    assert (np.abs(fewer.T @ X - Y.T @ X) > room).any()
    # row after row in float32, part after part
    total, left = np.zeros((n, d), np.float32), Y.copy()
    for q in range(f8_parts.COUNT[dtype]):
        part = f8_parts.upper_parts(torch.as_tensor(left), dtype, 1).numpy()
        left = left - part
        for t in range(m):
            total += np.float32(part[t][:, None] * X[t][None, :])
    assert (np.abs(total - Y.T @ X) <= room).all()


@pytest.mark.parametrize("m,n,d", PRODUCTS)
def test_a_product_that_is_cut_is_out_of_the_room(m, n, d):
    rng = np.random.default_rng([m, n, d])
    A, B = held(rng, m, d), held(rng, n, d)
    room = f8_rooms.product_room(A, B, torch.float32)
    assert (np.abs(f8_rooms.cut_products(A, B) - A @ B.T) > room).any()
    total = np.zeros((m, n), np.float32)
    for k in range(d):
        total += np.float32(np.outer(A[:, k], B[:, k]))
    assert (np.abs(total - A @ B.T) <= room).all()
