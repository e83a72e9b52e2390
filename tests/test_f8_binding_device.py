"""On which GPU and stream the calls on 8-bit matrices run and which workspaces they take, without a GPU: CPU tensors that say
that they lie on GPU 1, a library that notes the current GPU and the stream it is given, and GPU 0 current."""
import pytest

torch = pytest.importorskip("torch")

from test_binding_device import OnGpu0, OnGpu1, gpu1, stream_of  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    """(efanna_f8, list that receives (name, current GPU, arguments) of every call into the library, [current GPU])"""
    from paper_1609_07228_amd import efanna, efanna_f8
    current, made = [0], []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                if name.endswith("_workspace_bytes"):
                    return 512
                made.append((name, current[0], args))
                return 0
            self.__dict__[name] = entry          # (as ctypes does: argument types are set on it)
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
    yield efanna_f8, made, current


def table(f8, n=4, d=40):
    return f8.F8Table(gpu1(n, 128, dtype=torch.float8_e4m3fn), gpu1(n, 4, dtype=torch.uint8), d)


CALLS = {
    "efanna_f8_quantise": lambda f8, ws: f8.efanna_f8_quantise(gpu1(4, 40)),
    "efanna_f8_weights": lambda f8, ws: f8.efanna_f8_weights(gpu1(4, 40)),
    "efanna_f8_rows": lambda f8, ws: f8.efanna_f8_rows(table(f8), gpu1(3, dtype=torch.int32)),
    "efanna_f8_product": lambda f8, ws: f8.efanna_f8_product(table(f8), table(f8), workspace=ws),
    "efanna_f8_gradient": lambda f8, ws: f8.efanna_f8_gradient(gpu1(4, 7), table(f8), workspace=ws),
}


def test_every_call_is_here():
    from paper_1609_07228_amd import efanna_f8
    assert set(CALLS) == {s for s in efanna_f8.SYMBOLS if not s.endswith("_bytes")}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("here", [0, 1])
def test_runs_on_the_gpu_of_its_tensors(calls, name, here):
    f8, made, current = calls
    current[0] = here
    CALLS[name](f8, None)
    assert [(n, gpu, args[-1]) for n, gpu, args in made] == [(name, 1, stream_of(1))]
    assert current[0] == here


@pytest.mark.parametrize("name", ["efanna_f8_product", "efanna_f8_gradient"])
def test_workspace_lies_with_the_tensors_and_in_one_piece(calls, name):
    f8, made, _ = calls
    room = torch.zeros(4096, dtype=torch.uint8)
    for bad in (room, room.as_subclass(OnGpu0), room.as_subclass(OnGpu1)[::2]):
        with pytest.raises(ValueError):
            CALLS[name](f8, bad)
    assert made == []
    CALLS[name](f8, room.as_subclass(OnGpu1))
    assert made[0][2][-3:-1] == (room.data_ptr(), 4096)
    made.clear()
    CALLS[name](f8, torch.zeros(1024).as_subclass(OnGpu1))           # of another type: its bytes count
    assert made[0][2][-2] == 4096


def test_rows_that_are_further_apart(calls):
    f8, made, _ = calls
    f8.efanna_f8_quantise(gpu1(4, 50)[:, :40])
    f8.efanna_f8_weights(gpu1(4, 50)[:, :40])
    f8.efanna_f8_product(table(f8), table(f8, 6), out=gpu1(4, 9, dtype=torch.bfloat16)[:, :6])
    f8.efanna_f8_gradient(gpu1(4, 9)[:, :7], table(f8), out=gpu1(7, 44)[:, :40])
    args = {n: a for n, _, a in made}
    assert args["efanna_f8_quantise"][4] == args["efanna_f8_weights"][4] == 50
    assert args["efanna_f8_product"][11] == 9
    assert args["efanna_f8_gradient"][4] == 9 and args["efanna_f8_gradient"][11] == 44
