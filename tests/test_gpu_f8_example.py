"""The example that trains a projection with the operators on 8-bit tables: it runs, and its layer's gradients are the formulas'."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import f8_reference as ref  # noqa: E402


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: there is no CPU fallback")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "f8_projection.py")
    spec = importlib.util.spec_from_file_location("f8_projection", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,d", [(7, 5, 40), (300, 130, 257)])
def test_gradients_of_the_layer(example, dtype, m, n, d):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((m, d), generator=gen, device="cuda").to(dtype).requires_grad_()
    w = torch.randn((n, d), generator=gen, device="cuda").requires_grad_()
    dy = torch.randn((m, n), generator=gen, device="cuda").to(dtype)
    y = example.F8Linear.apply(x, w)
    y.backward(dy)
    X = ref.held(*ref.quantise(ref.host(x), "e4m3"), d, "e4m3")
    W = ref.held(*ref.quantise(ref.host(w), "e4m3", 128), d, "e4m3")
    G = ref.held(*ref.quantise(ref.host(dy), "e5m2"), n, "e5m2")
    Y = ref.host(dy)
    assert x.grad.dtype == dtype and w.grad.dtype == torch.float32
    assert (np.abs(ref.host(y) - X @ W.T) <= ref.product_room(X, W, dtype)).all()
    assert (np.abs(ref.host(x.grad) - G @ W) <= ref.product_room(G, W.T, dtype)).all()
    assert (np.abs(ref.host(w.grad) - Y.T @ X) <= ref.gradient_room(Y, X, torch.float32)).all()


def test_a_gradient_that_is_broadcast(example):
    """The gradient of a sum is one number for all results: rows that are one row in memory."""
    x = torch.ones((9, 40), device="cuda", requires_grad=True)
    w = torch.ones((6, 40), device="cuda", requires_grad=True)
    example.F8Linear.apply(x, w).sum().backward()
    assert torch.equal(w.grad, torch.full((6, 40), 9.0, device="cuda")) and torch.equal(x.grad, torch.full((9, 40), 6.0, device="cuda"))


def test_only_what_is_asked_for(example):
    x = torch.ones((9, 40), device="cuda")
    w = torch.ones((6, 40), device="cuda", requires_grad=True)
    example.F8Linear.apply(x, w).sum().backward()
    assert torch.equal(w.grad, torch.full((6, 40), 9.0, device="cuda")) and x.grad is None


def test_gradients_of_gradients_are_refused(example):
    x = torch.ones((9, 40), device="cuda", requires_grad=True)
    w = torch.ones((6, 40), device="cuda", requires_grad=True)
    dx, = torch.autograd.grad(example.F8Linear.apply(x, w).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


def test_a_captured_step_with_its_backward_pass(example):
    """Replayed several times with eager work between; inputs change in place."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((600, 200), generator=gen, device="cuda").requires_grad_()
    w = torch.randn((70, 200), generator=gen, device="cuda").requires_grad_()

    def step(x, w):
        y = example.F8Linear.apply(x, w)
        return (y.detach(), *torch.autograd.grad(y, (x, w), y.detach().sign()))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step(x, w)
    for _ in range(4):
        with torch.no_grad():
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            w.copy_(torch.randn(w.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        want = step(x.detach().clone().requires_grad_(), w.detach().clone().requires_grad_())
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_example_runs_as_a_whole(example):
    got = example.run("gmm10k_d32", 3000, 16, 5, 200)
    assert set(got) == {"before", "after"} and all(0.0 <= v <= 1.0 for v in got.values())
