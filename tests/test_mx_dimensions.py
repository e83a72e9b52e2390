"""Numbers that the entry points on MXFP4 tables take as 32-bit arguments: 2^32 + 5 coordinates are not five, and 2^32 + 1 neighbours not
one.  The binding refuses them as the library refuses what is too large.  Tensors without memory that say that they lie on the GPU."""
import pytest

torch = pytest.importorskip("torch")

from test_f8_dimensions import on_gpu  # noqa: E402


def table(ef, n, d):
    nb = (d + 31) // 32
    return ef.MxTable(on_gpu(n, 16 * nb, dtype=torch.uint8), on_gpu(n, (nb + 3) // 4 * 4, dtype=torch.uint8), on_gpu(n, dtype=torch.float32), d)


def calls(ef, d, k):
    yield lambda: ef.efanna_mx_quantise(on_gpu(1, d))
    yield lambda: ef.efanna_mx_rows(table(ef, 1, d))
    yield lambda: ef.efanna_mx_product(table(ef, 1, d), table(ef, 2, d))
    yield lambda: ef.efanna_mx_nearest(table(ef, 1, d), table(ef, 2, d), 1)
    yield lambda: ef.efanna_mx_nearest(table(ef, 1, 40), table(ef, 2, 40), k)


@pytest.mark.parametrize("d,k", [(65537, 129), (2 ** 31, 2 ** 31), (2 ** 32 + 5, 2 ** 32 + 1), (2 ** 33 + 64, -2 ** 32 + 1)])
def test_what_does_not_fit_an_argument_is_refused(monkeypatch, d, k):
    from paper_1609_07228_amd import build, efanna
    if build.stale():
        build.build()
    reached = []

    def call(name, on, *args):          # as the library would see it, and refuse it
        reached.append(args)
        raise efanna.EfannaError(-1, name)

    monkeypatch.setattr(efanna, "_call", call)
    monkeypatch.setattr(efanna, "_workspace", lambda need, on, given: on_gpu(1))
    for one in calls(efanna, d, k):
        with pytest.raises(efanna.EfannaError) as error:
            one()
        assert error.value.status == -1
    assert all(abs(a) < 2 ** 31 for args in reached for a in args if a in (d, k))
