"""The example that runs the operators on MXFP4 tables together with the graph's."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx_neighbours.py")
    spec = importlib.util.spec_from_file_location("mx_neighbours", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_graph_by_comparison_is_exact_where_the_format_is(example):
    """Coordinates that MXFP4 holds exactly: the table's neighbours are the set's."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randint(-3, 4, (700, 40), generator=gen, device="cuda").to(torch.float32)
    X[:, ::32] = 4.0                                     # every block's scale is 1
    ids, dists = example.graph_by_comparison(X, example.efanna.efanna_mx_quantise(X), 9, 0)
    dist = (X[:, None, :] - X[None, :, :]).square().sum(dim=2)
    dist.fill_diagonal_(torch.inf)
    key = dist.to(torch.float64) * 4096 + torch.arange(700, device="cuda")
    want = key.topk(9, dim=1, largest=False).indices
    assert torch.equal(ids.to(torch.int64), want)
    assert torch.equal(dists, dist.gather(1, want))


def test_example_runs_as_a_whole(example):
    got = example.run("gmm10k_d32", 4000, 10, 30, 64)
    assert set(got) == {"graph", "refined", "search", "spread", "score"}
    # refinement only replaces an entry by a nearer one
    assert 0.0 < got["graph"] <= got["refined"] <= 1.0
    assert got["search"] > 0.0 and got["spread"] > 0.0


def test_fewer_vectors_than_neighbours(example):
    X = torch.eye(5, 33, device="cuda")
    ids, dists = example.graph_by_comparison(X, example.efanna.efanna_mx_quantise(X), 6, 2)
    assert (ids[:, :4] >= 0).all() and (ids[:, 4:] == -1).all()
    assert (dists[:, :4] == 2.0).all() and torch.isinf(dists[:, 4:]).all()
