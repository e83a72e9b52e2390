"""Dimensions that the entry points on 8-bit matrices do not take are refused by the binding, with the reason, before anything is made:
they are 32-bit arguments, and 2^32 + 5 coordinates are not five.  Tensors without memory that say that they lie on the GPU."""
import pytest

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)


def table(f8, n, d):
    nb = (d + 127) // 128
    return f8.F8Table(on_gpu(n, 128 * nb, dtype=torch.float8_e4m3fn), on_gpu(n, (nb + 3) // 4 * 4, dtype=torch.uint8), d)


@pytest.fixture
def f8(monkeypatch):
    """The binding with a library that notes its calls (`f8.made`)."""
    from paper_1609_07228_amd import efanna_f8
    made, empty = [], torch.empty

    class Library:
        def __getattr__(self, name):
            return lambda *args: 0

    monkeypatch.setattr(efanna_f8, "lib", lambda: Library())
    monkeypatch.setattr(efanna_f8._efanna, "_call", lambda name, on, *args: made.append((name, args)))
    monkeypatch.setattr(efanna_f8._efanna.torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnGpu))
    monkeypatch.setattr(efanna_f8, "made", made, raising=False)
    return efanna_f8


def calls(f8, large):
    """Every call with a dimension of `large`."""
    yield lambda: f8.efanna_f8_quantise(on_gpu(1, large))
    yield lambda: f8.efanna_f8_weights(on_gpu(1, large))
    yield lambda: f8.efanna_f8_weights(on_gpu(large, 1))
    yield lambda: f8.efanna_f8_rows(table(f8, 1, large))
    yield lambda: f8.efanna_f8_product(table(f8, 1, large), table(f8, 2, large))
    yield lambda: f8.efanna_f8_gradient(on_gpu(1, large), table(f8, 1, 40))
    yield lambda: f8.efanna_f8_gradient(on_gpu(1, 40), table(f8, 1, large))


@pytest.mark.parametrize("large", [65537, 2 ** 31, 2 ** 32 + 5, 2 ** 33 + 128])
def test_larger_dimensions_are_refused_with_the_reason(f8, large):
    for call in calls(f8, large):
        with pytest.raises(ValueError, match="65536"):
            call()
    assert f8.made == []


def test_the_largest_dimension_goes_through(f8):
    for call in calls(f8, f8.MAX_D):
        call()
    assert len(f8.made) == 7 and all(f8.MAX_D in args for _, args in f8.made)
