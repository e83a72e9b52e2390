"""What the tests of the gradient's parts rest on, without a GPU: their shapes reach every tile of every type of dY, alone and in parts of the
sum, and their results differ if a part of dY is left out."""
import pytest

torch = pytest.importorskip("torch")

import f8_parts  # noqa: E402
from test_f8_launches import launches, numbers  # noqa: E402,F401
from test_mx_launches import BASE, OUT  # noqa: E402

TILES = {(4, 2, 2, 4): "square", (4, 2, 1, 8): "wide", (2, 2, 2, 2): "small", (1, 2, 2, 2): "narrow"}


def test_which_tile_each_shape_takes(launches):  # noqa: F811
    calls = [("efanna_f8_gradient", (BASE, t, m, n, n + 5, BASE, BASE, 0, d, 0, OUT, d, BASE, 1 << 40, None))
             for m, n, d in f8_parts.SHAPES for t in range(3)]
    got = [TILES[numbers(a["launches"][0]["symbol"])[1:5]] + " parts" * (len(a["launches"]) - 1) for a in launches(calls)]
    assert {s: tuple(got[3 * i:3 * i + 3]) for i, s in enumerate(f8_parts.SHAPES)} == f8_parts.SHAPES
    for t in range(3):
        assert {taken[t].split()[0] for taken in f8_parts.SHAPES.values()} == set(TILES.values())


@pytest.mark.parametrize("dtype", f8_parts.BITS)
def test_results_are_exact_and_need_every_part(dtype):
    m, n, d = 33, 260, 500
    Y, X = f8_parts.numbers(dtype, m, n, d, "cpu")
    assert torch.equal(Y.to(f8_parts.TYPES[dtype]).to(torch.float64), Y)
    want = Y.T @ X
    assert torch.equal(want.to(torch.float32).to(torch.float64), want)
    assert want.abs().max() < 2.0 ** 22 and torch.equal((want * 4).round(), want * 4)      # quarters, of 24 bits at most
    count = f8_parts.COUNT[dtype]
    assert torch.equal(f8_parts.upper_parts(Y, dtype, count), Y)
    for fewer in range(1, count):
        other = f8_parts.upper_parts(Y, dtype, fewer).T @ X
        assert (other != want).float().mean() > 0.5


@pytest.mark.parametrize("dtype", f8_parts.BITS)
def test_special_values_are_where_they_are_meant_to_be(dtype):
    m, n, d = 33, 260, 500
    Y, X, _, want = f8_parts.special(dtype, m, n, d, "cpu")
    nan = want.isnan()
    assert nan[0].all() and nan[:, d - 2].all() and nan[:, 128:256].all()
    assert nan.sum() < 0.4 * n * d
    inf = want.isinf()
    assert (inf | nan)[n - 1].all() and (inf | nan)[:, d - 1].all() and (inf | nan)[:, 3].all()
    assert nan[:, d - 1].any() and inf[:, d - 1].any()                # zeros of dY against an infinity, and numbers
    fine = want[want.isfinite()]
    assert len(fine) > 0.5 * n * d and torch.equal(fine.to(torch.float32).to(torch.float64), fine)
