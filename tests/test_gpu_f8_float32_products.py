"""Products of 8-bit tables to float32 add as float32 does, in every tile and every kernel for few rows: exact sums of large and small products,
and random numbers within a random walk's room."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_large_and_small  # noqa: E402
import f8_reference as ref  # noqa: E402
import f8_rooms  # noqa: E402
from f8_reference import FORMS, host  # noqa: E402
from test_gpu_f8 import SHAPES, matrix  # noqa: E402
from test_gpu_f8_tiles import PRODUCT_SHAPES  # noqa: E402

MIXED = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")]


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


@pytest.mark.parametrize("m,n,d", SHAPES + PRODUCT_SHAPES)
def test_small_products_next_to_large_ones(ef, m, n, d):
    A, B = f8_large_and_small.numbers(m, n, d)
    want = torch.as_tensor(A @ B.T).to(torch.float32).cuda()
    A, B = (torch.as_tensor(V).to(torch.float32).cuda() for V in (A, B))
    for a_form, b_form in MIXED:
        a, b = ef.efanna_f8_quantise(A, FORMS[a_form]), ef.efanna_f8_quantise(B, FORMS[b_form])
        assert torch.equal(ef.efanna_f8_product(a, b, dtype=torch.float32), want)


@pytest.mark.parametrize("m,n,d", SHAPES + [(2817, 3001, 600), (3000, 1300, 9000), (600, 300, 20_000), (20, 5000, 5000), (700, 20, 5000)])
def test_random_numbers(ef, m, n, d):
    rng = np.random.default_rng([4, m, n, d])
    for a_form, b_form in MIXED if m * n * d < 10 ** 9 else MIXED[1:2]:
        a = ef.efanna_f8_quantise(matrix(rng, m, d, "gauss"), FORMS[a_form])
        b = ef.efanna_f8_quantise(matrix(rng, n, d, "gauss"), FORMS[b_form])
        A, B = ref.held_by(a), ref.held_by(b)
        got = host(ef.efanna_f8_product(a, b, dtype=torch.float32))
        assert (np.abs(got - A @ B.T) <= f8_rooms.product_room(A, B, torch.float32)).all()
