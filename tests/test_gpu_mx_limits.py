"""MXFP4 tables at the limits that the header states: squared lengths next to the largest that have neighbours, more rows
than one launch takes; and long tables, whose groups of rows are so large that a wave takes them in several rounds."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna
    return efanna


# Squares of one block's values in units of 2^120 (scale 2^60, largest value 6): 64 of them are 2^126, 256 are 2^128.
JUST_BELOW = [6, 4, 3, 1.5, 0.5, 0.5]                 # 63.75: the nearest squared length below
JUST_AT = [6, 4, 3, 1.5, 0.5, 0.5, 0.5]               # 64
NEAR_THE_END = [6] * 7 + [1.5, 0.5, 0.5, 0.5]         # 255: finite in float32
BEYOND = [6] * 7 + [2]                                # 256: infinite


def rows(kinds, signs=None):
    x = np.zeros((len(kinds), 32), np.float32)
    for i, kind in enumerate(kinds):
        x[i, :len(kind)] = np.array(kind, np.float32) * np.float32(2.0) ** 60
        if signs is not None:
            x[i] *= signs[i]
    return x


@pytest.mark.parametrize("nq", [1, 40, 200])
@pytest.mark.parametrize("d", [32, 1100])
def test_rows_and_queries_on_both_sides_of_the_largest_norm(ef, nq, d):
    """Everything is a whole number of 2^118, so distances are exact."""
    kinds = [JUST_BELOW, JUST_AT, [0], NEAR_THE_END, [6], BEYOND, [0.5], JUST_BELOW, [-6], JUST_AT]
    x = np.zeros((len(kinds) * 30, d), np.float32)
    x[:, :32] = np.tile(rows(kinds), (30, 1))
    x[::7, :32] *= -1
    if d > 32:
        x[5::11, 1056:1088] = x[5::11, :32]           # the same in a block of its own, at the end of the row
        x[5::11, :32] = 0
    y = np.concatenate([x[:13], x[-7:]])
    y = np.tile(y, (nq // len(y) + 1, 1))[:nq]
    t, q = ef.efanna_mx_quantise(torch.from_numpy(x).cuda()), ef.efanna_mx_quantise(torch.from_numpy(y).cuda())
    X, Q = x.astype(np.float64), y.astype(np.float64)
    assert np.array_equal(ef.efanna_mx_rows(t).cpu().numpy(), x)          # the format holds them
    xx, qq = (X * X).sum(axis=1), (Q * Q).sum(axis=1)
    with np.errstate(over="ignore"):
        assert np.array_equal(t.norms.cpu().numpy(), xx.astype(np.float32))
    limit = ef.MX_MAX_NORM
    assert {0.0, limit * 63.75 / 64, limit, limit * 255 / 64} <= set(xx)
    ids, dists = (o.cpu().numpy() for o in ef.efanna_mx_nearest(t, q, 128))
    near = np.nonzero(xx < limit)[0]
    assert len(near) > 128 and (xx >= limit).any()
    for i in range(nq):
        if not qq[i] < limit:
            assert (ids[i] == -1).all() and np.isinf(dists[i]).all()
            continue
        dist = qq[i] + xx[near] - 2 * (X[near] @ Q[i])
        by = np.argsort(dist, kind="stable")[:128]
        assert np.array_equal(ids[i], near[by])
        assert np.array_equal(dists[i].astype(np.float64), dist[by])


def repeated(ef, d, n, dtype):
    """1009 rows, their table, and for n rows which of them each is."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((1009, d), generator=gen, device="cuda").to(dtype)
    return x, ef.efanna_mx_quantise(x), torch.arange(n, device="cuda", dtype=torch.int32) % 1009


def test_more_rows_than_one_launch_quantises(ef):
    """Rows of nine blocks take a wave each: 2^25 of them and some."""
    x, small, which = repeated(ef, 257, 2 ** 25 + 37, torch.bfloat16)
    t = ef.efanna_mx_quantise(x[which])
    assert torch.equal(t.norms, small.norms[which])
    assert torch.equal(t.scales, small.scales[which])
    assert torch.equal(t.codes, small.codes[which])


@pytest.mark.parametrize("by_id", [True, False])
def test_more_rows_than_one_launch_reads(ef, by_id):
    """Sixteen rows of 257 values a workgroup: 2^27 of them and some, 69 GB."""
    _, small, which = repeated(ef, 257, 2 ** 27 + 21, torch.bfloat16)
    if by_id:
        out = ef.efanna_mx_rows(small, which, factor=0.5, dtype=torch.bfloat16)
    else:
        table = ef.MxTable(small.codes[which], small.scales[which], small.norms[which], 257)
        out = ef.efanna_mx_rows(table, factor=0.5, dtype=torch.bfloat16)
    want = ef.efanna_mx_rows(small, factor=0.5, dtype=torch.bfloat16)
    assert out.shape == (len(which), 257)
    step = 2 ** 24
    for at in range(0, len(which), step):
        assert torch.equal(out[at:at + step], want[which[at:at + step]])


@pytest.mark.parametrize("first", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("nq", [3, 100])
def test_a_table_cut_from_any_row(ef, first, nq):
    """Every operator on rows `first` and on of a table, as views of it, and on a table of those rows alone."""
    gen = torch.Generator(device="cuda").manual_seed(first + nq)
    x = torch.randn((1000, 70), generator=gen, device="cuda")
    whole, alone = ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(x[first:])
    cut = ef.MxTable(whole.codes[first:], whole.scales[first:], whole.norms[first:], 70)
    q = ef.efanna_mx_quantise(torch.randn((nq, 70), generator=gen, device="cuda"))
    for got, want in zip(ef.efanna_mx_nearest(cut, q, 9), ef.efanna_mx_nearest(alone, q, 9)):
        assert torch.equal(got, want)
    for got, want in zip(ef.efanna_mx_nearest(q, cut, 2), ef.efanna_mx_nearest(q, alone, 2)):
        assert torch.equal(got, want)
    assert torch.equal(ef.efanna_mx_rows(cut), ef.efanna_mx_rows(alone))
    assert torch.equal(ef.efanna_mx_product(q, cut), ef.efanna_mx_product(q, alone))
    assert torch.equal(ef.efanna_mx_product(cut, q), ef.efanna_mx_product(alone, q))


@pytest.mark.parametrize("n,d", [(250_003, 16), (262_144, 128), (110_001, 200), (440_001, 256), (300_007, 500), (75_003, 600),
                                 (292_001, 640), (130_001, 896), (125_009, 1000), (492_007, 1024)])
@pytest.mark.parametrize("nq", [1, 40, 130, 600])
def test_groups_of_rows_that_take_several_rounds(ef, n, d, nq):
    """The shapes next above those from which groups of 32, 64 and 128 rows are taken for one neighbour."""
    gen = torch.Generator(device="cuda").manual_seed(n + nq)
    x = torch.randint(-2, 3, (n, d), generator=gen, device="cuda").to(torch.float32)
    y = torch.randint(-2, 3, (nq, d), generator=gen, device="cuda").to(torch.float32)
    x[:, ::32], y[:, ::32] = 4.0, 4.0                    # every block's scale is 1
    t, q = ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y)
    xx = x.square().sum(dim=1)
    for _ in range(2):
        ids, dists = ef.efanna_mx_nearest(t, q, 1)
        for at in list(range(min(nq, 40))) + [nq - 1]:
            dist = (xx - 2.0 * (x @ y[at]) + y[at].square().sum()).to(torch.float64)       # whole numbers below 2^24
            want = (dist * 2 ** 20 + torch.arange(n, device="cuda")).argmin()
            assert ids[at, 0] == want and dists[at, 0] == dist[want]


@pytest.mark.parametrize("power", [-55, -63, -66, -73])
@pytest.mark.parametrize("m,n,d", [(3, 300, 64), (300, 301, 256), (20, 100, 1100)])
def test_products_below_the_normal_range(ef, power, m, n, d):
    """Small whole multiples of a power whose square is subnormal or next to it: nothing is lost above 2^-149."""
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    x = torch.randint(-2, 3, (m, d), generator=gen, device="cuda").to(torch.float64)
    y = torch.randint(-2, 3, (n, d), generator=gen, device="cuda").to(torch.float64)
    x[:, ::32], y[:, ::32] = 4.0, 4.0
    a, b = (ef.efanna_mx_quantise((v * 2.0 ** power).to(torch.float32)) for v in (x, y))
    product = x @ y.T
    assert torch.equal(ef.efanna_mx_product(a, b).to(torch.float64), product * 2.0 ** (2 * power))
    dist = x.square().sum(dim=1, keepdim=True) + y.square().sum(dim=1) - 2 * product
    want = (dist * 4096 + torch.arange(n, device="cuda")).topk(7, dim=1, largest=False).indices
    ids, dists = ef.efanna_mx_nearest(b, a, 7)
    assert torch.equal(ids.to(torch.int64), want)
    assert torch.equal(dists.to(torch.float64), dist.gather(1, want) * 2.0 ** (2 * power))
