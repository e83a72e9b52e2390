"""On which GPU and stream the binding's calls run, which workspaces they take and what they hand over of a table cut out of
another, without a GPU: CPU tensors that say that they lie on GPU 1, a library that notes the current GPU and the stream it is
given, and GPU 0 current."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


class OnGpu1(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1


def gpu1(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu1)


def stream_of(gpu):
    return 1000 + gpu


@pytest.fixture
def calls(monkeypatch):
    """(efanna, list that receives (name, current GPU, last argument) of every call into the library)"""
    from paper_1609_07228_amd import efanna
    current, made = [0], []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                if name.endswith("_workspace_bytes"):
                    return 512
                made.append((name, current[0], args[-1]))
                return 0
            return entry

    class On:
        def __init__(self, gpu):
            self.gpu = gpu if isinstance(gpu, int) else gpu.index

        def __enter__(self):
            self.before, current[0] = current[0], self.gpu

        def __exit__(self, *_):
            current[0] = self.before

    library, empty = Library(), torch.empty
    monkeypatch.setattr(efanna, "lib", lambda: library)
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", stream_of)
    # what the binding makes beside its arguments lies there too
    monkeypatch.setattr(efanna.torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnGpu1))
    yield efanna, made, current


def table(ef, n=4, d=40):
    return ef.MxTable(gpu1(n, 32, dtype=torch.uint8), gpu1(n, 4, dtype=torch.uint8), gpu1(n), d)


CALLS = {
    "efanna_build_trees": lambda ef: ef.efanna_build_trees(gpu1(9, 4), 2, 4, 0),
    "efanna_build_trees_rule": lambda ef: ef.efanna_build_trees_rule(gpu1(9, 4), 2, 4, 0, ef.SPLIT_VARIANCE),
    "efanna_init_graph": lambda ef: ef.efanna_init_graph(gpu1(9, 4), gpu1(2, 9, dtype=torch.int32),
                                                         gpu1(2, 10, dtype=torch.int32), np.ones(2, np.int32), 4, 3),
    "efanna_nndescent": lambda ef: ef.efanna_nndescent(gpu1(9, 4), gpu1(9, 3, dtype=torch.int64), 1, 4, 0),
    "efanna_nndescent_noalloc": lambda ef: ef.efanna_nndescent_noalloc(gpu1(9, 4), gpu1(9, 3, dtype=torch.int64), 1, 4, 0,
                                                                       gpu1(1, 4, dtype=torch.int64)),
    "efanna_get_graph": lambda ef: ef.efanna_get_graph(gpu1(9, 3, dtype=torch.int64)),
    "efanna_set_graph": lambda ef: ef.efanna_set_graph(gpu1(9, 3, dtype=torch.int32), gpu1(9, 3)),
    "efanna_pair_distances": lambda ef: ef.efanna_pair_distances(gpu1(9, 4), gpu1(5, dtype=torch.int32),
                                                                 gpu1(5, dtype=torch.int32)),
    "efanna_search": lambda ef: ef.efanna_search(gpu1(9, 4), gpu1(2, 9, dtype=torch.int32), gpu1(2, 10, dtype=torch.int32),
                                                 np.ones(2, np.int32), gpu1(2, 10, 32, dtype=torch.uint8), 1, 4,
                                                 gpu1(9, 3, dtype=torch.int32), gpu1(2, 4), 1, 4, 2, 1),
    "efanna_mx_quantise": lambda ef: ef.efanna_mx_quantise(gpu1(4, 40)),
    "efanna_mx_rows": lambda ef: ef.efanna_mx_rows(table(ef)),
    "efanna_mx_product": lambda ef: ef.efanna_mx_product(table(ef), table(ef)),
    "efanna_mx_nearest": lambda ef: ef.efanna_mx_nearest(table(ef), table(ef), 2),
}


def test_every_call_is_here():
    from paper_1609_07228_amd import efanna
    assert set(CALLS) == {s for s in efanna.SYMBOLS if not s.endswith("_bytes") and s != "efanna_status_string"}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("here", [0, 1])
def test_runs_on_the_gpu_of_its_tensors(calls, name, here):
    efanna, made, current = calls
    current[0] = here
    CALLS[name](efanna)
    assert made == [(name, 1, stream_of(1))]
    assert current[0] == here


TAKES_WORKSPACE = {
    "efanna_build_trees": lambda ef, ws: ef.efanna_build_trees(gpu1(9, 4), 2, 4, 0, workspace=ws),
    "efanna_init_graph": lambda ef, ws: ef.efanna_init_graph(gpu1(9, 4), gpu1(2, 9, dtype=torch.int32),
                                                             gpu1(2, 10, dtype=torch.int32), np.ones(2, np.int32), 4, 3,
                                                             workspace=ws),
    "efanna_nndescent": lambda ef, ws: ef.efanna_nndescent(gpu1(9, 4), gpu1(9, 3, dtype=torch.int64), 1, 4, 0, workspace=ws),
    "efanna_search": lambda ef, ws: ef.efanna_search(gpu1(9, 4), gpu1(2, 9, dtype=torch.int32), gpu1(2, 10, dtype=torch.int32),
                                                     np.ones(2, np.int32), gpu1(2, 10, 32, dtype=torch.uint8), 1, 4,
                                                     gpu1(9, 3, dtype=torch.int32), gpu1(2, 4), 1, 4, 2, 1, workspace=ws),
    "efanna_mx_nearest": lambda ef, ws: ef.efanna_mx_nearest(table(ef), table(ef), 2, workspace=ws),
}


class OnGpu0(OnGpu1):
    def get_device(self):
        return 0


@pytest.mark.parametrize("name", TAKES_WORKSPACE)
def test_workspace_lies_with_the_tensors_and_in_one_piece(calls, name):
    """A kernel would write wherever the pointer leads: host memory, another GPU, or what lies between a view's elements."""
    efanna, made, _ = calls
    room = torch.zeros(4096, dtype=torch.uint8)
    for bad in (room, room.as_subclass(OnGpu0), room.as_subclass(OnGpu1)[::2]):
        with pytest.raises(ValueError):
            TAKES_WORKSPACE[name](efanna, bad)
    assert made == []
    TAKES_WORKSPACE[name](efanna, room.as_subclass(OnGpu1))
    assert len(made) == 1


@pytest.mark.parametrize("first", range(6))
def test_norms_of_a_table_cut_from_any_row(calls, monkeypatch, first):
    """The entry point asks for norms at a multiple of 16 bytes; codes and scales are at one from any row on."""
    efanna, _, _ = calls
    import ctypes
    seen = []

    def call(name, on, codes, scales, norms, n, *rest):
        seen.append((codes, scales, norms % 16, list((ctypes.c_float * n).from_address(norms))))
    monkeypatch.setattr(efanna, "_call", call)
    whole = efanna.MxTable(gpu1(9, 32, dtype=torch.uint8), gpu1(9, 4, dtype=torch.uint8),
                           torch.arange(9, dtype=torch.float32).as_subclass(OnGpu1), 40)
    cut = efanna.MxTable(whole.codes[first:], whole.scales[first:], whole.norms[first:], 40)
    efanna.efanna_mx_nearest(cut, whole, 2)
    assert seen == [(cut.codes.data_ptr(), cut.scales.data_ptr(), 0, [float(i) for i in range(first, 9)])]
