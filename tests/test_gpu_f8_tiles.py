"""8-bit matrices on the GPU at sizes that take the larger tiles, many tiles, and sums in parts: whole numbers, whose results are exact,
against products in float64."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from f8_reference import FORMS, TYPES  # noqa: E402

# (rows, columns of dY, coordinates)
GRADIENT_SHAPES = [(500, 1000, 1030), (500, 1000, 2050), (1500, 90, 4000), (500, 2300, 4000), (12_000, 90, 4000), (1500, 2300, 2050),
                   (4000, 2000, 2050), (12_000, 1030, 1000), (60_000, 128, 1000), (60_001, 128, 1000), (60_000, 60, 200), (8000, 90, 1000),
                   (4001, 2003, 2049), (100_000, 128, 960), (100_000, 65, 960), (3001, 1100, 1301)]
# (rows of a, rows of b, coordinates)
PRODUCT_SHAPES = [(3000, 2900, 100), (3000, 1300, 9000), (2817, 3001, 600), (33, 9000, 1100), (9000, 40, 1100), (1100, 1300, 640),
                  (20, 700, 5000), (700, 20, 5000), (20, 5000, 5000), (4100, 4100, 129), (600, 300, 20_000), (10, 300, 5000), (300, 30, 300),
                  (25, 300, 300), (256, 256, 65_536)]


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


def whole(gen, n, d, most):
    return torch.randint(-most, most + 1, (n, d), generator=gen, device="cuda").to(torch.float32)


def powers(gen, n, most):
    return torch.exp2(torch.randint(-most, most + 1, (n, 1), generator=gen, device="cuda").to(torch.float32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,d", GRADIENT_SHAPES)
def test_gradient(ef, dtype, m, n, d):
    gen = torch.Generator(device="cuda").manual_seed(m + n + d)
    size = powers(gen, m, 3)
    X, Y = whole(gen, m, d, 2) * size, whole(gen, m, n, 9) / size
    for form in FORMS.values():
        x = ef.efanna_f8_quantise(X, form)
        for out in TYPES.values():
            got = ef.efanna_f8_gradient(Y.to(TYPES[dtype]), x, dtype=out)
            assert torch.equal(got, (Y.double().T @ X.double()).to(torch.float32).to(out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,d", PRODUCT_SHAPES)
def test_product(ef, dtype, m, n, d):
    gen = torch.Generator(device="cuda").manual_seed(m + n + d)
    each = powers(gen, (d + 127) // 128, 4).repeat_interleave(128)[:d]
    rows = powers(gen, m, 3)
    A, B = whole(gen, m, d, 2) * each * rows, whole(gen, n, d, 2) / each
    want = (A.double() @ B.double().T).to(torch.float32).to(TYPES[dtype])
    for a_form, b_form in (("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")):
        a, b = ef.efanna_f8_quantise(A, FORMS[a_form]), ef.efanna_f8_quantise(B, FORMS[b_form])
        assert torch.equal(ef.efanna_f8_product(a, b, dtype=TYPES[dtype]), want)
