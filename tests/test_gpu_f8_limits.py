"""8-bit matrices on the GPU at their limits: tables past 4 GB of codes, results past 2^31 elements, scales that stand for NaN, rows and
columns that end anywhere, two graphs at once."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_reference as ref  # noqa: E402
from f8_reference import FORMS, TYPES, host  # noqa: E402


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


LONG = 33_600_000                 # rows of 128 bytes: past 2^32 bytes


@pytest.fixture(scope="module")
def long_table(ef):
    """(a table of zeros but for its last 70 rows, these as numbers)"""
    rng = np.random.default_rng(5)
    last = rng.integers(-2, 3, (70, 100)).astype(np.float32)
    t = ef.efanna_f8_quantise(torch.as_tensor(last).cuda())
    codes = torch.zeros((LONG, 128), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((LONG, 4), dtype=torch.uint8, device="cuda")
    codes[-70:], scales[-70:] = t.codes.view(torch.uint8), t.scales
    yield ef.F8Table(codes.view(torch.float8_e4m3fn), scales, 100), last
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [20, 64])
def test_products_with_a_long_table(ef, long_table, dtype, m):
    """Few rows and tiles; 64 x 33.6 * 10^6 results are past 2^31."""
    t, last = long_table
    rng = np.random.default_rng(6)
    q = rng.integers(-2, 3, (m, 100)).astype(np.float32)
    a = ef.efanna_f8_quantise(torch.as_tensor(q).cuda())
    want = host(torch.as_tensor(q @ last.T).to(dtype))
    got = ef.efanna_f8_product(a, t, dtype=dtype)
    assert np.array_equal(host(got[:, -70:]), want) and not got[:, :-70].any()
    del got
    got = ef.efanna_f8_product(t, a, dtype=dtype)
    assert np.array_equal(host(got[-70:]), want.T) and not got[:-70].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_of_a_long_table(ef, long_table, dtype):
    t, last = long_table
    dy = torch.zeros((LONG, 9), dtype=TYPES[dtype], device="cuda")
    tail = torch.randint(-9, 10, (70, 9), generator=torch.Generator().manual_seed(1)).to(TYPES[dtype])
    dy[-70:] = tail.cuda()
    dy[:1000] = 3.0                                        # (against rows of zeros)
    assert np.array_equal(host(ef.efanna_f8_gradient(dy, t)), host(tail).T @ last)


@pytest.mark.parametrize("m,n", [(5, 40), (40, 5), (50, 60)])
def test_a_scale_that_stands_for_nan(ef, m, n):
    """Whatever its codes are, zeros too."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    a, b = (ef.efanna_f8_quantise(torch.randn((k, 300), generator=gen, device="cuda")) for k in (m, n))
    a.scales[3, 1] = 255
    a.codes.view(torch.uint8)[3, 128:200] = 0
    assert np.array_equal(np.isnan(host(ef.efanna_f8_rows(a))), np.isnan(ref.held_by(a)))
    for dtype in TYPES.values():
        got = ef.efanna_f8_product(a, b, dtype=dtype)
        assert got[3].isnan().all() and got.isnan().sum() == n
        got = ef.efanna_f8_product(b, a, dtype=dtype)
        assert got[:, 3].isnan().all() and got.isnan().sum() == n
        got = ef.efanna_f8_gradient(torch.randn((m, 20), generator=gen, device="cuda").to(dtype), a)
        assert got[:, 128:256].isnan().all() and got.isnan().sum() == 20 * 128


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 15, 127, 129, 135, 255, 257, 263, 513])
def test_gradient_reads_nothing_behind_its_columns(ef, dtype, n):
    """dY is cut out of a matrix of NaN, down to its last element."""
    rng = np.random.default_rng(n)
    for m in (1, 31, 32, 33, 200):
        pad = 5
        wide = torch.full((m * (n + pad) + 3,), float("nan"), dtype=TYPES[dtype], device="cuda")
        dy = wide[3:].view(m, n + pad)[:, :n]
        Y = rng.integers(-9, 10, (m, n)).astype(np.float64)
        dy.copy_(torch.as_tensor(Y))
        X = rng.integers(-2, 3, (m, 150)).astype(np.float32)
        x = ef.efanna_f8_quantise(torch.as_tensor(X).cuda())
        assert np.array_equal(host(ef.efanna_f8_gradient(dy, x)), Y.T @ X)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [1, 7, 8, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513])
def test_rows_end_anywhere(ef, dtype, d):
    """Rows between rows of NaN, quantised both ways and read back into a guarded place."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    wide = torch.full((37, d + 9), float("nan"), dtype=TYPES[dtype], device="cuda")
    x = wide[:, 4:4 + d]
    x.copy_(torch.randn((37, d), generator=gen, device="cuda"))
    for form in FORMS:
        t = ef.efanna_f8_quantise(x, FORMS[form])
        codes, scales = ref.quantise(host(x), form)
        assert np.array_equal(host(t.codes), codes) and np.array_equal(host(t.scales), scales)
        w, turned = ef.efanna_f8_weights(x, FORMS[form])
        codes, scales = ref.quantise(host(x), form, 128)
        assert np.array_equal(host(w.codes), codes) and np.array_equal(host(w.scales), scales)
        assert np.array_equal(ref.held_by(turned), ref.held_by(w).T)


def test_two_graphs_at_once(ef):
    """Graphs of calls that need workspaces, replayed in turn and on two streams at once."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    sets, graphs, kept, want = [], [], [], []
    for i in range(2):
        a, b = (ef.efanna_f8_quantise(torch.randn((k, 6000), generator=gen, device="cuda")) for k in (50 + i, 200))
        dy, x = torch.randn((5000, 60 + i), generator=gen, device="cuda"), ef.efanna_f8_quantise(torch.randn((5000, 300), generator=gen, device="cuda"))
        assert ef.lib().efanna_f8_product_workspace_bytes(50 + i, 200, 6000, 2) and ef.lib().efanna_f8_gradient_workspace_bytes(5000, 60 + i, 300, 0)
        sets.append((a, b, dy, x))
        want.append((ef.efanna_f8_product(a, b), ef.efanna_f8_gradient(dy, x)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept.append((ef.efanna_f8_product(a, b), ef.efanna_f8_gradient(dy, x)))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for k, w in zip(kept, want):
            assert all(torch.equal(p, q) for p, q in zip(k, w))
            for t in k:
                t.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("m,n,d", [(40, 50, 20_000), (33, 33, 65_536), (300, 200, 9000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_long_sums_in_parts(ef, m, n, d, dtype):
    rng = np.random.default_rng(d)
    A = rng.integers(-2, 3, (m, d)) * (rng.random((m, d)) < 0.004)
    B = rng.integers(-2, 3, (n, d))
    a, b = (ef.efanna_f8_quantise(torch.as_tensor(v).to(torch.float32).cuda()) for v in (A, B))
    got = ef.efanna_f8_product(a, b, dtype=TYPES[dtype])
    assert np.array_equal(host(got), host(torch.as_tensor((A @ B.T).astype(np.float64)).to(TYPES[dtype])))
