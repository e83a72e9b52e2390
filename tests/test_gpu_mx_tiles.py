"""Products of MXFP4 tables with more tiles than run at once, a workgroup for each, with sums of one stage to several and remainders
in every direction.  Coordinates are whole numbers that the format holds, so every output is known exactly."""
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
@pytest.mark.parametrize("m,n,d", [(4300, 4500, 32), (4352, 4608, 290), (4300, 4608, 512), (4352, 4500, 960), (4300, 4500, 1568),
                                   (4352, 8704, 2048), (3000, 3000, 32), (2944, 3000, 288), (3001, 2999, 1000), (2944, 2944, 1280)])
def test_products_of_many_tiles(ef, dtype, m, n, d):
    x, y = whole_numbers(m, d, m + d), whole_numbers(n, d, n + d + 1)
    a, b = ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y)
    want = (x.to(torch.float64) @ y.to(torch.float64).T).to(dtype)          # below 2^24: float32 sums are exact too
    for _ in range(3):
        assert torch.equal(ef.efanna_mx_product(a, b, dtype=dtype), want)


def test_rows_apart_and_not_aligned(ef):
    m, n, d = 4300, 4500, 320
    x, y = whole_numbers(m, d, 1), whole_numbers(n, d, 2)
    wide = torch.full((m, n + 13), 5.0, dtype=torch.float16, device="cuda")
    out = wide[:, 3:3 + n]
    ef.efanna_mx_product(ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y), dtype=torch.float16, out=out)
    assert torch.equal(out, (x.to(torch.float64) @ y.to(torch.float64).T).to(torch.float16))
    assert (wide[:, :3] == 5).all() and (wide[:, 3 + n:] == 5).all()
