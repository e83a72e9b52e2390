"""Products of MXFP4 tables on both sides of where tiles of 128 x 128 give way to tiles of 256 x 256 (512 of the small ones), and of
few rows to either.  Coordinates are whole numbers that the format holds, so every output is known exactly."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna
    return efanna


def whole_numbers(n, d, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-2, 3, (n, d), generator=gen, device="cuda").to(torch.float32)
    x[:, ::32] = 4.0                          # every block's scale is 1
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,d", [(2816, 2800, 290), (2816, 2800, 1000), (2800, 2816, 2048), (4096, 2048, 33), (2048, 4096, 1313),
                                   (4097, 2048, 1000), (33, 65536, 544), (33, 65537, 544), (8192, 8, 960), (65536, 129, 256),
                                   (32, 8192, 8192), (33, 8192, 8192), (1000, 8191, 512)])
def test_products_around_the_choice_of_tiles(ef, dtype, m, n, d):
    x, y = whole_numbers(m, d, m + d), whole_numbers(n, d, n + d + 1)
    a, b = ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y)
    want = (x.to(torch.float64) @ y.to(torch.float64).T).to(dtype)          # below 2^24: float32 sums are exact too
    for _ in range(3):
        assert torch.equal(ef.efanna_mx_product(a, b, dtype=dtype), want)
