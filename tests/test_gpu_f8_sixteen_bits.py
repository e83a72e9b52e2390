"""Products of 8-bit tables to 16 bits where what the 8-bit instructions cut off adds up: terms of one sign, terms of very different size.  Within
the bound that efanna_f8.h states, never too large where all terms are positive but for the rounding, and the same bits every time."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_reference as ref  # noqa: E402
from f8_reference import FORMS, host  # noqa: E402

SHAPES = [(3, 70, 300), (16, 300, 4096), (32, 100, 960), (50, 60, 300), (300, 515, 1025), (1100, 1300, 640), (2817, 3001, 300)]


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


def numbers(rng, kind, n, d):
    x = rng.standard_normal((n, d))
    return np.abs(x) if kind == "positive" else np.exp(2 * x) if kind == "uneven" else np.exp(2 * x) * rng.choice([-1.0, 1.0], (n, d))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", ["positive", "uneven", "uneven signs"])
@pytest.mark.parametrize("m,n,d", SHAPES)
def test_products(ef, dtype, kind, m, n, d):
    rng = np.random.default_rng([8, m, n, d])
    for a_form, b_form in (("e4m3", "e4m3"), ("e5m2", "e4m3")):
        # (scaled so that sums are within half precision's range)
        a = ef.efanna_f8_quantise(torch.as_tensor(numbers(rng, kind, m, d) / (64 * d)).to(torch.float32).cuda(), FORMS[a_form])
        b = ef.efanna_f8_quantise(torch.as_tensor(numbers(rng, kind, n, d)).to(torch.float32).cuda(), FORMS[b_form])
        A, B = ref.held_by(a), ref.held_by(b)
        got, want = ef.efanna_f8_product(a, b, dtype=dtype), A @ B.T
        assert np.abs(want).max() < 60_000
        assert (np.abs(host(got) - want) <= ref.product_room(A, B, dtype)).all()
        if kind != "uneven signs":          # cut towards zero: only sums and the result are rounded up
            up = (d + 8) * 2.0 ** -23 * want
            assert (host(got) - want <= up + (want + up) * ref.HALF_STEP[dtype] + ref.LEAST[dtype]).all()
        for _ in range(3):
            assert torch.equal(ef.efanna_f8_product(a, b, dtype=dtype), got)
