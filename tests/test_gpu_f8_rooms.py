"""Gradients of random numbers on the GPU against 64 bits within bounds that a part of dY left out would break."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_parts  # noqa: E402
import f8_reference as ref  # noqa: E402
import f8_rooms  # noqa: E402
from f8_reference import FORMS, TYPES, host  # noqa: E402
from test_gpu_f8 import GRADIENT_SHAPES, matrix  # noqa: E402

LARGE = [(33, 2051, 3900), (1500, 2304, 2050), (500, 1000, 2050), (12_000, 1030, 1000)]


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,d", GRADIENT_SHAPES + LARGE)
def test_gradient(ef, dtype, m, n, d):
    rng = np.random.default_rng([3, m, n, d])
    for form in FORMS if m * n * d < 10 ** 9 else ["e4m3"]:
        dy = matrix(rng, m, n, "gauss", TYPES[dtype], 3)
        x = ef.efanna_f8_quantise(matrix(rng, m, d, "gauss"), FORMS[form])
        Y, X = host(dy), ref.held_by(x)
        got = host(ef.efanna_f8_gradient(dy, x))
        assert (np.abs(got - Y.T @ X) <= f8_rooms.gradient_room(Y, X, f8_parts.COUNT[dtype], torch.float32)).all()
