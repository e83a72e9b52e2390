"""What the entry points on 8-bit matrices refuse, their symbols and their workspaces: found on the host, before anything is
launched, so no GPU is needed."""
import ctypes as C
import os
import re

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

EINVAL, EWORKSPACE, EUNSUPPORTED, OK = -1, -2, -6, 0
ONE = C.c_void_p(4096)          # never dereferenced: every call below fails, or has nothing to do
ODD = C.c_void_p(4097)
HALF = C.c_void_p(4098)
EIGHT = C.c_void_p(4104)


@pytest.fixture(scope="module")
def f8():
    from paper_1609_07228_amd import build
    if build.stale():
        build.build()
    from paper_1609_07228_amd import efanna_f8
    return efanna_f8


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "efanna_f8.h")).read(), flags=re.S)


def test_every_declared_symbol_is_exported_and_bound(f8):
    protos = dict(re.findall(r"\b(efanna_f8_[a-z_0-9]+)\s*\(([^)]*)\)\s*;", header()))
    assert set(protos) == set(f8.SYMBOLS)
    for name, args in protos.items():
        assert len(getattr(f8.lib(), name).argtypes) == len(args.split(",")), name


def test_limits_are_the_same_in_header_and_binding(f8):
    assert int(re.search(r"#define EFANNA_F8_MAX_D (\d+)", header()).group(1)) == f8.MAX_D


def refuses(f, ok, bad, status=EINVAL):
    for one in bad:
        assert f(*{**ok, **one}.values()) == status, one


def test_quantise(f8):
    f = f8.lib().efanna_f8_quantise
    ok = dict(X=ONE, dtype=0, n=10, d=40, ldx=40, form=0, codes=ONE, scales=ONE, stream=None)
    refuses(f, ok, (dict(X=None), dict(codes=None), dict(scales=None), dict(dtype=3), dict(dtype=-1), dict(form=2), dict(form=-1),
                    dict(n=-1), dict(n=2 ** 31 - 65536), dict(d=0), dict(d=65537), dict(ldx=39), dict(codes=EIGHT),
                    dict(scales=HALF), dict(X=HALF), dict(X=ODD, dtype=1)))
    assert f(*{**ok, **dict(n=0, X=None, codes=None, scales=None)}.values()) == OK


def test_weights(f8):
    f = f8.lib().efanna_f8_weights
    ok = dict(W=ONE, dtype=0, n=10, d=40, ldw=40, form=0, codes=ONE, scales=ONE, t_codes=ONE, t_scales=ONE, stream=None)
    refuses(f, ok, (dict(W=None), dict(codes=None), dict(scales=None), dict(t_codes=None), dict(t_scales=None), dict(dtype=3),
                    dict(form=2), dict(n=-1), dict(n=65537), dict(d=0), dict(d=65537, ldw=65537), dict(ldw=39),
                    dict(codes=EIGHT), dict(scales=HALF), dict(t_codes=EIGHT), dict(t_scales=HALF), dict(W=HALF),
                    dict(W=ODD, dtype=2)))
    assert f(*{**ok, **dict(n=0, W=None, codes=None, scales=None)}.values()) == OK


def test_rows(f8):
    f = f8.lib().efanna_f8_rows
    ok = dict(codes=ONE, scales=ONE, form=0, n=10, d=40, ids=ONE, m=5, factor=1.0, dtype=0, out=ONE, stream=None)
    refuses(f, ok, (dict(codes=None), dict(scales=None), dict(out=None), dict(dtype=7), dict(form=2), dict(n=-1), dict(d=0),
                    dict(d=65537), dict(m=-1), dict(ids=None, m=11), dict(out=HALF), dict(out=ODD, dtype=2), dict(ids=HALF),
                    dict(codes=ODD), dict(scales=ODD), dict(m=2 ** 31)))
    assert f(*{**ok, **dict(m=0, out=None, ids=None)}.values()) == OK
    assert f(*{**ok, **dict(m=0, n=0, codes=None, scales=None, out=None)}.values()) == OK


def test_product(f8):
    L = f8.lib()
    m, n, d = 40, 100, 40_000
    need = L.efanna_f8_product_workspace_bytes(m, n, d, 0)
    ok = dict(ac=ONE, asc=ONE, af=0, m=m, bc=ONE, bsc=ONE, bf=1, n=n, d=d, dtype=0, out=ONE, ldo=n, ws=ONE, size=need, stream=None)
    refuses(L.efanna_f8_product, ok,
            (dict(ac=None), dict(asc=None), dict(bc=None), dict(bsc=None), dict(out=None), dict(m=-1), dict(n=-1), dict(d=0),
             dict(d=65537), dict(dtype=3), dict(af=2), dict(bf=-1), dict(ldo=n - 1), dict(out=HALF), dict(out=ODD, dtype=1),
             dict(ac=ODD), dict(bc=EIGHT), dict(asc=HALF), dict(bsc=HALF), dict(n=2 ** 31, ldo=2 ** 31)))
    if need:
        refuses(L.efanna_f8_product, ok, (dict(ws=None), dict(ws=C.c_void_p(4096 + 16)), dict(size=need - 1)), EWORKSPACE)
    assert L.efanna_f8_product(*{**ok, **dict(m=0, ac=None, asc=None, out=None, ws=None, size=0)}.values()) == OK
    assert L.efanna_f8_product(*{**ok, **dict(n=0, ldo=0, bc=None, bsc=None, out=None, ws=None, size=0)}.values()) == OK


def test_gradient(f8):
    L = f8.lib()
    m, n, d = 100_000, 60, 40
    need = L.efanna_f8_gradient_workspace_bytes(m, n, d, 0)
    ok = dict(dy=ONE, dtype=0, m=m, n=n, ldy=n, codes=ONE, scales=ONE, form=0, d=d, out_dtype=0, out=ONE, ldo=d, ws=ONE, size=need,
              stream=None)
    refuses(L.efanna_f8_gradient, ok,
            (dict(dy=None), dict(codes=None), dict(scales=None), dict(out=None), dict(dtype=3), dict(out_dtype=-1), dict(form=2),
             dict(m=-1), dict(m=2 ** 31 - 65536), dict(n=-1), dict(n=65537, ldy=65537), dict(d=0), dict(d=65537, ldo=65537), dict(ldy=n - 1),
             dict(ldo=d - 1), dict(codes=EIGHT), dict(scales=HALF), dict(dy=HALF), dict(dy=ODD, dtype=1), dict(out=HALF),
             dict(out=ODD, out_dtype=2)))
    if need:
        refuses(L.efanna_f8_gradient, ok, (dict(ws=None), dict(ws=C.c_void_p(4096 + 16)), dict(size=need - 1)), EWORKSPACE)
    assert L.efanna_f8_gradient(*{**ok, **dict(ldy=2 ** 24)}.values()) == EUNSUPPORTED
    assert L.efanna_f8_gradient(*{**ok, **dict(n=0, ldy=0, dy=None, out=None, ws=None, size=0)}.values()) == OK


def test_workspace_sizes(f8):
    product, gradient = f8.lib().efanna_f8_product_workspace_bytes, f8.lib().efanna_f8_gradient_workspace_bytes
    for bad in ((-1, 1, 1, 0), (1, -1, 1, 0), (1, 1, 0, 0), (1, 1, 65537, 0), (2 ** 31, 1, 1, 0), (100, 100, 60000, 3)):
        assert product(*bad) == 0
    for bad in ((-1, 1, 1, 0), (1, -1, 1, 0), (1, 1, 0, 0), (1, 1, 65537, 0), (2 ** 31, 1, 1, 0), (1, 65537, 1, 0), (9999, 1, 1, 3)):
        assert gradient(*bad) == 0
    # parts of a sum are only as many as it takes to fill the GPU
    for m in (1, 40, 300, 5000, 2 ** 31 - 65537):
        for n in (1, 50, 4000, 65536):
            for d in (1, 300, 9000, 65536):
                assert all(product(m, n, d, dtype) <= 256 << 20 for dtype in range(3))
                if n <= 65536:
                    assert all(gradient(m, n, d, dtype) <= 256 << 20 for dtype in range(3))


def test_binding_checks_types_shapes_and_devices(f8):
    x = torch.zeros((4, 40))
    t = f8.F8Table(torch.zeros((4, 128), dtype=torch.float8_e4m3fn), torch.zeros((4, 4), dtype=torch.uint8), 40)
    for call in (lambda: f8.efanna_f8_quantise(x), lambda: f8.efanna_f8_quantise(x.to(torch.float64)),
                 lambda: f8.efanna_f8_quantise(x, torch.float16), lambda: f8.efanna_f8_weights(x),
                 lambda: f8.efanna_f8_rows(t), lambda: f8.efanna_f8_rows(t, dtype=torch.float64),
                 lambda: f8.efanna_f8_product(t, t), lambda: f8.efanna_f8_product(t, t, dtype=torch.int32),
                 lambda: f8.efanna_f8_gradient(x, t), lambda: f8.efanna_f8_gradient(x, t, dtype=torch.float64)):
        with pytest.raises(ValueError):
            call()


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


def table(f8, n, d, form=torch.float8_e4m3fn):
    nb = (d + 127) // 128
    return f8.F8Table(on_gpu(n, 128 * nb, dtype=form), on_gpu(n, (nb + 3) // 4 * 4, dtype=torch.uint8), d)


def test_binding_checks_what_belongs_together(f8, monkeypatch):
    """Tensors that say that they lie on the GPU, and no call that gets through."""
    def never(*a):
        raise AssertionError("the library was called")
    monkeypatch.setattr(f8._efanna, "_call", never)
    t = table(f8, 4, 300)
    bad_tables = (t._replace(codes=t.codes.to(torch.uint8).as_subclass(OnGpu)), t._replace(d=129), t._replace(scales=t.scales[:3]),
                  t._replace(scales=t.scales.to(torch.int32).as_subclass(OnGpu)), t._replace(codes=on_gpu(384, 4, dtype=torch.float8_e4m3fn).T),
                  t._replace(scales=on_gpu(4, 4, dtype=torch.uint8).T))
    for bad in bad_tables:
        for call in (lambda: f8.efanna_f8_rows(bad), lambda: f8.efanna_f8_product(bad, t), lambda: f8.efanna_f8_product(t, bad),
                     lambda: f8.efanna_f8_gradient(on_gpu(4, 5), bad)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: f8.efanna_f8_quantise(on_gpu(4, 5).T), lambda: f8.efanna_f8_quantise(on_gpu(4)),
                 lambda: f8.efanna_f8_weights(on_gpu(4, 5).T), lambda: f8.efanna_f8_rows(t, on_gpu(3, dtype=torch.int64)),
                 lambda: f8.efanna_f8_product(t, table(f8, 4, 301)), lambda: f8.efanna_f8_product(t, t, out=on_gpu(4, 5)),
                 lambda: f8.efanna_f8_product(t, t, out=on_gpu(4, 4)),                     # bfloat16 is expected
                 lambda: f8.efanna_f8_product(t, t, dtype=torch.float32, out=on_gpu(4, 8)[:, ::2]),
                 lambda: f8.efanna_f8_gradient(on_gpu(5, 6), t), lambda: f8.efanna_f8_gradient(on_gpu(6, 4).T, t),
                 lambda: f8.efanna_f8_gradient(on_gpu(4, 6), t, out=on_gpu(6, 301))):
        with pytest.raises(ValueError):
            call()
