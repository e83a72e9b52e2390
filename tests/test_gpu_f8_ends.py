"""Products and gradients of 8-bit tables whose values lie at the ends of float32's range, as efanna_f8.h states them: below 2^-126 they
count in steps of 2^-133 in float32 products and gradients, and exactly in products to 16 bits; 2^128 is an infinity."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_parts  # noqa: E402
import f8_reference as ref  # noqa: E402
import f8_rooms  # noqa: E402
from f8_reference import FORMS, TYPES, host  # noqa: E402

STEP = 2.0 ** -133
# few rows, tiles, and rows of more than one block
SHAPES = [(5, 40, 128), (40, 5, 300), (50, 60, 300), (33, 300, 1100)]


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


def table(ef, rng, n, d, form, scales):
    """Random codes with scale bytes taken from `scales`."""
    nb = (d + 127) // 128
    codes = rng.integers(0, 127 if form == "e4m3" else 124, (n, nb * 128)) | rng.integers(0, 2, (n, nb * 128)) << 7
    codes[:, d:] = 0
    bytes_ = np.zeros((n, (nb + 3) // 4 * 4), np.uint8)
    bytes_[:, :nb] = rng.choice(scales, (n, nb))
    return ef.F8Table(torch.as_tensor(codes.astype(np.uint8)).cuda().view(FORMS[form]), torch.as_tensor(bytes_).cuda(), d)


# scale bytes of tables with values around 2^-126 and far below, and of what they are multiplied with: results are within half precision's range
SMALL = {"e4m3": ([0, 1, 2, 6], [238]), "e5m2": ([0, 1, 2, 6], [231])}


def loses_if_flushed(A, B, room):
    """(the test would see values below 2^-126 taken as zeros)"""
    return (np.abs(np.where(np.abs(A) < 2.0 ** -126, 0.0, A) @ B.T - A @ B.T) > room).any()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("m,n,d", SHAPES)
def test_small_values_in_products(ef, form, m, n, d):
    rng = np.random.default_rng([m, n, d])
    a, b = table(ef, rng, m, d, form, SMALL[form][0]), table(ef, rng, n, d, form, SMALL[form][1])
    A, B = ref.held_by(a), ref.held_by(b)
    room = f8_rooms.product_room(A, B, torch.float32) + STEP * (np.abs(A) < 2.0 ** -126).astype(np.float64) @ np.abs(B).T
    assert loses_if_flushed(A, B, room)
    assert (np.abs(host(ef.efanna_f8_product(a, b, dtype=torch.float32)) - A @ B.T) <= room).all()
    assert (np.abs(host(ef.efanna_f8_product(b, a, dtype=torch.float32)).T - A @ B.T) <= room).all()
    for dtype in (torch.float16, torch.bfloat16):
        assert (np.abs(host(ef.efanna_f8_product(a, b, dtype=dtype)) - A @ B.T) <= ref.product_room(A, B, dtype)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_small_values_of_the_table_in_gradients(ef, form, dtype):
    for m, n, d in ((40, 30, 300), (300, 70, 200), (33, 501, 4100)):
        rng = np.random.default_rng([m, n, d])
        x = table(ef, rng, m, d, form, SMALL[form][0])
        dy = torch.as_tensor(rng.standard_normal((m, n)) * 2.0 ** (10 if dtype == "f16" else 110)).to(TYPES[dtype]).cuda()
        Y, X = host(dy), ref.held_by(x)
        room = f8_rooms.gradient_room(Y, X, f8_parts.COUNT[dtype], torch.float32) + STEP * np.abs(Y).T @ (np.abs(X) < 2.0 ** -126).astype(np.float64)
        assert loses_if_flushed(X.T, Y.T, room.T)
        assert (np.abs(host(ef.efanna_f8_gradient(dy, x)) - Y.T @ X) <= room).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_values_of_dy_in_gradients(ef, dtype):
    """Down to the smallest numbers: parts below 2^-133 are lost, which bfloat16 numbers do not have."""
    for m, n, d in ((40, 30, 300), (300, 70, 200), (33, 501, 4100)):
        rng = np.random.default_rng([m, n, d, 1])
        x = table(ef, rng, m, d, "e4m3", [238])
        dy = torch.as_tensor(rng.standard_normal((m, n)) * np.exp2(rng.integers(-135, -115, (m, n)))).to(TYPES[dtype]).cuda()
        Y, X = host(dy), ref.held_by(x)
        room = f8_rooms.gradient_room(Y, X, f8_parts.COUNT[dtype], torch.float32)
        assert loses_if_flushed(Y.T, X.T, room)
        if dtype == "f32":
            room = room + STEP * np.ones_like(Y).T @ np.abs(X)
        assert (np.abs(host(ef.efanna_f8_gradient(dy, x)) - Y.T @ X) <= room).all()


@pytest.mark.parametrize("form", FORMS)
def test_two_to_the_128(ef, form):
    largest = torch.full((40, 200), torch.finfo(torch.float32).max, device="cuda")
    largest[:, 1:] = 0.0
    a = ef.efanna_f8_quantise(largest, FORMS[form])
    assert ref.held_by(a)[0, 0] == 2.0 ** 128
    assert torch.equal(ef.efanna_f8_rows(a)[:, 0], torch.full((40,), float("inf"), device="cuda"))
    small = torch.full((50, 200), 2.0 ** -20, device="cuda")
    small[3] = 0.0
    b = ef.efanna_f8_quantise(small, FORMS[form])
    for rows in (slice(0, 5), slice(0, 50)):
        part = ef.F8Table(b.codes[rows], b.scales[rows], 200)
        got = ef.efanna_f8_product(a, part, dtype=torch.float32)
        assert got[:, 3].isnan().all() and got[:, :3].isposinf().all()
        got = ef.efanna_f8_product(a, part, dtype=torch.bfloat16)
        assert got[:, 3].eq(0.0).all() and got[:, :3].eq(2.0 ** 108).all()
    dy = torch.full((40, 70), 2.0 ** -20, device="cuda")
    dy[:, 3] = 0.0
    for dtype in TYPES.values():
        got = ef.efanna_f8_gradient(dy.to(dtype), a)
        assert got[3, 0].isnan() and got[:3, 0].isposinf().all() and got[:, 1:].eq(0.0).all()
