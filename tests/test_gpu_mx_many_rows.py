"""Nearest rows of MXFP4 tables so long that many groups of rows stand to be chosen from, all of them equally good or nearly so."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ef():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    from paper_1609_07228_amd import efanna
    return efanna


@pytest.mark.parametrize("n", [140_001, 262_144, 300_007])
@pytest.mark.parametrize("k", [1, 40, 128])
@pytest.mark.parametrize("nq", [3, 300, 2100])
def test_equal_rows_go_by_id(ef, n, k, nq):
    t = ef.efanna_mx_quantise(torch.full((n, 8), 1.5, device="cuda"))
    q = ef.efanna_mx_quantise(torch.full((nq, 8), 1.5, device="cuda"))
    ids, dists = ef.efanna_mx_nearest(t, q, k)
    assert torch.equal(ids, torch.arange(k, dtype=torch.int32, device="cuda").expand(nq, k)) and (dists == 0).all()


@pytest.mark.parametrize("n,k", [(300_007, 128), (300_007, 20), (140_001, 33)])
@pytest.mark.parametrize("nq", [2, 300, 2100])
def test_few_different_distances(ef, n, k, nq):
    """Two coordinates of few whole numbers: distances are exact, hundreds of rows share each."""
    gen = torch.Generator(device="cuda").manual_seed(n + k + nq)
    x = torch.randint(-4, 5, (n, 2), generator=gen, device="cuda").to(torch.float32)
    x[x.abs() == 5] = 4.0
    y = x[torch.randint(0, n, (nq,), generator=gen, device="cuda")].contiguous()
    t, q = ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y)
    X, Q = ef.efanna_mx_rows(t), ef.efanna_mx_rows(q)
    ids, dists = ef.efanna_mx_nearest(t, q, k)
    row = torch.arange(n, device="cuda")
    for i in list(range(min(nq, 24))) + [nq - 1]:
        dist = (X - Q[i]).square().sum(dim=1).to(torch.float64)
        want = (dist * 2 ** 20 + row).topk(k, largest=False).indices        # (distance, id): 2^20 is more than the rows
        assert torch.equal(ids[i].to(torch.int64), want)
        assert torch.equal(dists[i].to(torch.float64), dist[want])


@pytest.mark.parametrize("d", [640, 768, 800, 960, 1024])
@pytest.mark.parametrize("nq", [16, 17, 40, 64, 65])
def test_long_rows_and_tens_of_queries(ef, d, nq):
    """Whole numbers, so that sums are exact; the last group is not full."""
    gen = torch.Generator(device="cuda").manual_seed(d + nq)
    n, k = 2777, 12
    x = torch.randint(-2, 3, (n, d), generator=gen, device="cuda").to(torch.float32)
    y = torch.randint(-2, 3, (nq, d), generator=gen, device="cuda").to(torch.float32)
    x[:, ::32], y[:, ::32] = 4.0, 4.0                    # every block's scale is 1
    ids, dists = ef.efanna_mx_nearest(ef.efanna_mx_quantise(x), ef.efanna_mx_quantise(y), k)
    X, Q = x.to(torch.float64), y.to(torch.float64)
    dist = Q.square().sum(dim=1, keepdim=True) + X.square().sum(dim=1) - 2 * (Q @ X.T)
    want = (dist * 4096 + torch.arange(n, device="cuda")).topk(k, dim=1, largest=False).indices
    assert torch.equal(ids.to(torch.int64), want)
    assert torch.equal(dists.to(torch.float64), dist.gather(1, want))
