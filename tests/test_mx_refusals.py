"""Argument errors of the MXFP4 entry points: found on the host, before anything is launched, so no
GPU is needed.  The binding's own checks (types, shapes, devices) run on CPU tensors."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

EINVAL, EWORKSPACE, OK = -1, -2, 0
ONE = C.c_void_p(4096)          # never dereferenced: every call below fails, or has nothing to do
ODD = C.c_void_p(4097)
HALF = C.c_void_p(4098)


@pytest.fixture(scope="module")
def efanna():
    from paper_1609_07228_amd import build
    if build.stale():
        build.build()
    from paper_1609_07228_amd import efanna
    return efanna


def test_quantise(efanna):
    f = efanna.lib().efanna_mx_quantise
    ok = dict(X=ONE, dtype=0, n=10, d=40, ldx=40, codes=ONE, scales=ONE, norms=ONE, stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())
    for bad in (dict(X=None), dict(codes=None), dict(scales=None), dict(norms=None), dict(dtype=3), dict(dtype=-1),
                dict(n=-1), dict(n=2 ** 31 - 65536), dict(d=0), dict(d=65537), dict(ldx=39), dict(codes=ODD),
                dict(codes=C.c_void_p(4104)), dict(scales=HALF), dict(norms=HALF), dict(X=HALF), dict(X=ODD, dtype=1)):
        assert call(**bad) == EINVAL, bad
    assert call(n=0, X=None, codes=None, scales=None, norms=None) == OK


def test_rows(efanna):
    f = efanna.lib().efanna_mx_rows
    ok = dict(codes=ONE, scales=ONE, n=10, d=40, ids=ONE, m=5, factor=1.0, dtype=0, out=ONE, stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())
    for bad in (dict(codes=None), dict(scales=None), dict(out=None), dict(dtype=7), dict(n=-1), dict(d=0), dict(d=65537),
                dict(m=-1), dict(ids=None, m=11), dict(out=HALF), dict(out=ODD, dtype=2), dict(ids=HALF), dict(codes=ODD),
                dict(scales=ODD), dict(m=2 ** 31)):
        assert call(**bad) == EINVAL, bad
    assert call(m=0, out=None, ids=None) == OK
    assert call(m=0, n=0, codes=None, scales=None, out=None) == OK


def test_product(efanna):
    f = efanna.lib().efanna_mx_product
    ok = dict(ac=ONE, asc=ONE, m=3, bc=ONE, bsc=ONE, n=7, d=64, dtype=0, out=ONE, ldo=7, stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())
    for bad in (dict(ac=None), dict(asc=None), dict(bc=None), dict(bsc=None), dict(out=None), dict(m=-1), dict(n=-1),
                dict(d=0), dict(d=65537), dict(dtype=3), dict(ldo=6), dict(out=HALF), dict(out=ODD, dtype=1), dict(ac=ODD),
                dict(bc=ODD), dict(asc=HALF), dict(bsc=HALF), dict(n=2 ** 31, ldo=2 ** 31)):
        assert call(**bad) == EINVAL, bad
    assert call(m=0, ac=None, asc=None, out=None) == OK
    assert call(n=0, bc=None, bsc=None, out=None, ldo=0) == OK


def test_nearest(efanna):
    L = efanna.lib()
    need = L.efanna_mx_nearest_workspace_bytes(1000, 64, 20, 5)
    assert need > 0
    ok = dict(c=ONE, s=ONE, x=ONE, n=1000, d=64, qc=ONE, qs=ONE, qx=ONE, nq=20, k=5, first_self=-1, ids=ONE, dists=ONE,
              ws=ONE, ws_bytes=need, stream=None)

    def call(**kw):
        return L.efanna_mx_nearest(*{**ok, **kw}.values())
    for bad in (dict(c=None), dict(s=None), dict(x=None), dict(qc=None), dict(qs=None), dict(qx=None), dict(ids=None),
                dict(dists=None), dict(n=-1), dict(nq=-1), dict(d=0), dict(d=65537), dict(k=0), dict(k=129), dict(c=ODD),
                dict(qc=ODD), dict(s=HALF), dict(qs=HALF), dict(x=C.c_void_p(4100)), dict(qx=HALF), dict(ids=HALF),
                dict(dists=ODD)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(ws=None), dict(ws=C.c_void_p(4352 + 16)), dict(ws_bytes=need - 1)):
        assert call(**bad) == EWORKSPACE, bad
    assert call(nq=0, qc=None, qs=None, qx=None, ids=None, dists=None, ws=None, ws_bytes=0) == OK


def test_workspace_sizes(efanna):
    need = efanna.lib().efanna_mx_nearest_workspace_bytes
    assert need(-1, 64, 1, 1) == need(1, 64, -1, 1) == need(1, 64, 1, 0) == need(1, 64, 1, 129) == 0
    assert need(2 ** 31, 64, 1, 1) == need(1, 0, 1, 1) == need(1, 65537, 1, 1) == 0
    assert 0 < need(0, 64, 0, 1) <= 4096
    assert need(1000, 64, 1, 1) <= need(100_000, 64, 1, 1) <= need(100_000, 64, 1000, 1)
    for n, d, nq, k in ((1_000_000, 128, 10_000, 10), (1_000_000, 960, 1_000_000, 10), (4_000_000, 96, 4_000_000, 100)):
        assert need(n, d, nq, k) <= (1 << 30) + (1 << 20)      # further queries take further passes


def test_binding_checks_types_shapes_and_devices(efanna):
    x = torch.zeros((4, 40))
    with pytest.raises(ValueError):
        efanna.efanna_mx_quantise(x)                                    # not on a device
    with pytest.raises(ValueError):
        efanna.efanna_mx_quantise(x.to(torch.float64))
    t = efanna.MxTable(torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8), torch.zeros(4), 40)
    for call in (lambda: efanna.efanna_mx_rows(t), lambda: efanna.efanna_mx_product(t, t),
                 lambda: efanna.efanna_mx_nearest(t, t, 2), lambda: efanna.efanna_mx_rows(t, dtype=torch.float64),
                 lambda: efanna.efanna_mx_product(t, t, dtype=torch.int32)):
        with pytest.raises(ValueError):
            call()
