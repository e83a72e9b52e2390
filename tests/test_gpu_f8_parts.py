"""The gradient of the weights in every tile of its kernel with numbers that fill all parts of dY (three of float32, two of half precision),
rows of dY further apart than they are long, and results that are exact; infinities, NaN and scales that stand for NaN in every tile."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_parts  # noqa: E402
from f8_reference import FORMS  # noqa: E402


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


@pytest.mark.parametrize("dtype", f8_parts.BITS)
@pytest.mark.parametrize("m,n,d", f8_parts.SHAPES)
def test_every_part_counts(ef, dtype, m, n, d):
    Y, X = f8_parts.numbers(dtype, m, n, d, "cuda")
    dy, want = f8_parts.cut_out(Y, dtype), (Y.T.contiguous() @ X).to(torch.float32)
    for form in FORMS.values():
        x = ef.efanna_f8_quantise(X.to(torch.float32), form)
        assert torch.equal(ef.efanna_f8_gradient(dy, x), want)
    assert torch.equal(ef.efanna_f8_gradient(dy, x, dtype=torch.bfloat16), want.to(torch.bfloat16))


@pytest.mark.parametrize("dtype", f8_parts.BITS)
@pytest.mark.parametrize("m,n,d", f8_parts.SHAPES)
def test_what_is_not_finite_stays_in_its_results(ef, dtype, m, n, d):
    Y, X, (row, block), want = f8_parts.special(dtype, m, n, d, "cuda")
    x = ef.efanna_f8_quantise(X.to(torch.float32), torch.float8_e5m2)
    x.scales[row, block] = 255
    got = ef.efanna_f8_gradient(f8_parts.cut_out(Y, dtype), x).to(torch.float64)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(torch.where(got.isnan(), 0.0, got), torch.where(want.isnan(), 0.0, want))

