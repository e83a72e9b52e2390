"""What the entry points on 8-bit matrices launch, up to the most rows that they accept, without a GPU: the HIP runtime's entry points
are taken by a stand-in that hands every launch to the test.  A launch takes fewer than 2^32 threads along an axis, and the launches
of a call together have to take every row once."""
import json
import re
import subprocess
import sys

import pytest

from test_mx_launches import BASE, MAX_ROWS, OUT, STAND_IN

CALLER = r"""
import ctypes as C, json, re, sys
stand_in, library, calls = sys.argv[1], sys.argv[2], json.loads(sys.argv[3])
S = C.CDLL(stand_in, mode=C.RTLD_GLOBAL)
names, made = {}, []
def value(args, i, t):
    return C.cast(args[i], C.POINTER(t))[0]
class Table(C.Structure):
    _fields_ = [("codes", C.c_uint64), ("scales", C.c_uint64), ("n", C.c_int), ("nb", C.c_int), ("sp", C.c_int)]
def on_launch(f, gx, gy, gz, bx, by, bz, args):
    name = re.search(r"(f8_[a-z_]+_kernel)", names[f].decode()).group(1)
    one = dict(kernel=name, grid=[gx, gy, gz], block=[bx, by, bz], symbol=names[f].decode())
    if name == "f8_quantise_kernel":
        one.update(x=value(args, 0, C.c_uint64), n=value(args, 1, C.c_uint32), group=value(args, 4, C.c_int),
                   codes=value(args, 7, C.c_uint64), scales=value(args, 8, C.c_uint64))
    elif name == "f8_rows_kernel":
        t = value(args, 0, Table)
        one.update(codes=t.codes, scales=t.scales, table_n=t.n, ids=value(args, 2, C.c_uint64), n=value(args, 3, C.c_int64),
                   group=value(args, 4, C.c_int), pieces=value(args, 5, C.c_int), out=value(args, 7, C.c_uint64))
    elif name == "f8_product_few_kernel":
        a, b = value(args, 0, Table), value(args, 1, Table)
        one.update(few=a.n, codes=b.codes, scales=b.scales, n=b.n, out=value(args, 3, C.c_uint64), step_a=value(args, 4, C.c_int64),
                   step_b=value(args, 5, C.c_int64))
    made.append(one)
launch_t = C.CFUNCTYPE(None, C.c_void_p, *[C.c_uint] * 6, C.POINTER(C.c_void_p))
register_t = C.CFUNCTYPE(None, C.c_void_p, C.c_char_p)
on_launch, on_register = launch_t(on_launch), register_t(lambda f, name: names.__setitem__(f, name))
S.stand_in(on_launch, on_register)
L = C.CDLL(library)
vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
L.efanna_f8_quantise.argtypes = [vp, i32, i64, i32, i64, i32, vp, vp, vp]
L.efanna_f8_weights.argtypes = [vp, i32, i32, i32, i64, i32, vp, vp, vp, vp, vp]
L.efanna_f8_rows.argtypes = [vp, vp, i32, i64, i32, vp, i64, C.c_float, i32, vp, vp]
L.efanna_f8_product.argtypes = [vp, vp, i32, i64, vp, vp, i32, i64, i32, i32, vp, i64, vp, sz, vp]
L.efanna_f8_gradient.argtypes = [vp, i32, i64, i32, i64, vp, vp, i32, i32, i32, vp, i64, vp, sz, vp]
answers = []
for name, args in calls:
    made.clear()
    status = getattr(L, name)(*args)
    answers.append(dict(status=status, launches=list(made)))
print(json.dumps(answers))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """Runs calls [(name, args)] and returns [{status, launches}]."""
    from paper_1609_07228_amd import build
    if build.stale():
        build.build()
    folder = tmp_path_factory.mktemp("launches")
    source, library = folder / "stand_in.c", folder / "stand_in.so"
    source.write_text(STAND_IN)
    subprocess.run(["gcc", "-w", "-shared", "-fPIC", "-o", str(library), str(source)], check=True)

    def run(calls):
        done = subprocess.run([sys.executable, "-c", CALLER, str(library), build.LIB, json.dumps(calls)], capture_output=True,
                              text=True, timeout=300)
        assert done.returncode == 0, done.stderr
        answers = json.loads(done.stdout.splitlines()[-1])
        for answer in answers:
            for one in answer["launches"]:
                assert all(g * b < 2 ** 32 and g < 2 ** 31 for g, b in zip(one["grid"], one["block"])), one
                assert one["grid"][1] <= 65535 and one["grid"][2] == 1
        return answers
    return run


COUNTS = [1, 1000, 2 ** 26, 2 ** 26 + 1, 2 ** 27 + 5, 2 ** 30 + 3, MAX_ROWS]


def pitches(d):
    nb = (d + 127) // 128
    return nb, (nb + 3) // 4 * 4


@pytest.mark.parametrize("d,group", [(1, 8), (64, 8), (65, 16), (128, 16), (200, 32), (257, 64), (1024, 64), (65536, 64)])
def test_quantise_takes_every_row_once(launches, d, group):
    nb, sp = pitches(d)
    words, ldx = sp // 4, d + 3
    for n, got in zip(COUNTS, launches([("efanna_f8_quantise", (BASE, 2, n, d, ldx, 0, 2 * BASE, 3 * BASE, None)) for n in COUNTS])):
        assert got["status"] == 0
        done = 0
        for one in got["launches"]:
            assert one["kernel"] == "f8_quantise_kernel" and one["block"] == [256, 1, 1] and one["group"] == group
            assert one["x"] == BASE + done * ldx * 2 and one["codes"] == 2 * BASE + done * nb * 128 and one["scales"] == 3 * BASE + done * sp
            assert one["n"] % words == 0 and one["grid"] == [-(-one["n"] // (256 // group)), 1, 1]
            done += one["n"] // words
        assert done == n


@pytest.mark.parametrize("ids", [None, 5 * BASE])
@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
@pytest.mark.parametrize("d", [1, 50, 300, 3000, 65536])
def test_rows_takes_every_row_once(launches, ids, dtype, size, d):
    nb, sp = pitches(d)
    counts = COUNTS + [2 ** 28, 2 ** 28 + 1]
    n = MAX_ROWS
    for m, got in zip(counts, launches([("efanna_f8_rows", (BASE, 2 * BASE, 1, n, d, ids, m, 1.0, dtype, OUT, None)) for m in counts])):
        assert got["status"] == 0
        done = 0
        for one in got["launches"]:
            assert one["kernel"] == "f8_rows_kernel" and one["block"] == [256, 1, 1]
            first = 0 if ids else done                      # row 0 of the table that the kernel is given
            assert one["codes"] == BASE + first * nb * 128 and one["scales"] == 2 * BASE + first * sp and one["table_n"] == n - first
            assert one["ids"] == (ids + done * 4 if ids else 0) and one["out"] == OUT + done * d * size
            assert one["pieces"] * one["group"] * 16 >= d * size > (one["pieces"] - 1) * one["group"] * 16
            per = 256 // one["group"]
            assert one["grid"][0] % one["pieces"] == 0
            rows = one["grid"][0] // one["pieces"]
            assert rows in (-(-one["n"] // per), -(-one["n"] // (4 * per)))
            done += one["n"]
        assert done == m


@pytest.mark.parametrize("d", [128, 500, 3000])
@pytest.mark.parametrize("few", [1, 17, 32])
@pytest.mark.parametrize("n", [33, 2 ** 27 + 5, MAX_ROWS])
@pytest.mark.parametrize("dtype,size", [(0, 4), (2, 2)])
def test_products_against_few_rows_take_every_row_once(launches, d, few, n, dtype, size):
    nb, sp = pitches(d)
    straight, turned = launches([("efanna_f8_product", (BASE, BASE, 0, few, 2 * BASE, 3 * BASE, 1, n, d, dtype, OUT, n + 2, None, 0, None)),
                                 ("efanna_f8_product", (2 * BASE, 3 * BASE, 0, n, BASE, BASE, 1, few, d, dtype, OUT, few + 2, None, 0, None))])
    for got, steps in ((straight, (n + 2, 1)), (turned, (1, few + 2))):
        assert got["status"] == 0
        done = 0
        for one in got["launches"]:
            assert one["kernel"] == "f8_product_few_kernel" and one["few"] == few
            assert (one["step_a"], one["step_b"]) == steps
            assert one["codes"] == 2 * BASE + done * nb * 128 and one["scales"] == 3 * BASE + done * sp
            assert one["out"] == OUT + done * steps[1] * size
            assert one["grid"][0] in (-(-one["n"] // 64), -(-one["n"] // 16))
            done += one["n"]
        assert done == n


@pytest.mark.parametrize("m,n,d,status", [(33, 33, 64, 0), (33, 2 ** 28, 64, 0), (2 ** 20, 2 ** 18, 64, 0), (2 ** 20, 2 ** 20, 64, -6),
                                          (2 ** 26, 2 ** 26, 64, -6), (5000, 300, 65536, 0)])
@pytest.mark.parametrize("dtype", [0, 2])
def test_products_are_launched_or_refused(launches, m, n, d, status, dtype):
    """Refused (EFANNA_EUNSUPPORTED) is only what would need half a terabyte."""
    got, = launches([("efanna_f8_product", (BASE, BASE, 0, m, BASE, BASE, 1, n, d, dtype, OUT, n, BASE, 1 << 40, None))])
    assert got["status"] == status
    assert bool(got["launches"]) == (status == 0)
    if status:
        assert m * n * 2 >= 2 ** 39


@pytest.mark.parametrize("n,d", [(1, 1), (65536, 1), (1, 65536), (65536, 65536), (128, 960), (1000, 3000)])
def test_gradients_and_weights_of_all_sizes(launches, n, d):
    for m in (0, 1, 100, 100_000, MAX_ROWS):
        got, = launches([("efanna_f8_gradient", (BASE, 0, m, n, n + 1, BASE, BASE, 0, d, 2, OUT, d, BASE, 1 << 40, None))])
        assert got["status"] == 0
        assert [one["kernel"] for one in got["launches"]] in (["f8_gradient_kernel"], ["f8_gradient_kernel", "f8_join_kernel"])
    got, = launches([("efanna_f8_weights", (BASE, 1, n, d, d, 1, BASE, BASE, BASE, BASE, None))])
    assert got["status"] == 0 and got["launches"][0]["grid"] == [(d + 127) // 128, (n + 127) // 128, 1]


def numbers(symbol):
    """A kernel's template arguments that are numbers."""
    return tuple(int(v) for v in re.findall(r"L[ib](\d+)E", symbol))


def test_every_kernel_runs_in_the_tests_of_results(launches):
    """The shapes that results are tested with reach every variant of every kernel, alone and in parts."""
    import test_gpu_f8 as small
    import test_gpu_f8_tiles as large
    gradients, products = {}, {}
    calls = [("efanna_f8_gradient", (BASE, t, m, n, n, BASE, BASE, 0, d, 0, OUT, d, BASE, 1 << 40, None))
             for t in range(3) for m, n, d in small.GRADIENT_SHAPES + large.GRADIENT_SHAPES]
    for (_, args), got in zip(calls, launches(calls)):
        gradients.setdefault(args[1], set()).add((numbers(got["launches"][0]["symbol"])[1:5], len(got["launches"])))
    for t in range(3):
        assert {tile for tile, _ in gradients[t]} == {(4, 2, 2, 4), (4, 2, 1, 8), (2, 2, 2, 2), (1, 2, 2, 2)}, t
        assert {parts for _, parts in gradients[t]} == {1, 2}
    calls = [("efanna_f8_product", (BASE, BASE, 0, m, BASE, BASE, 0, n, d, t, OUT, n, BASE, 1 << 40, None))
             for t in (0, 2) for m, n, d in small.SHAPES + large.PRODUCT_SHAPES]
    for (_, args), got in zip(calls, launches(calls)):
        one = got["launches"][0]
        products.setdefault(args[9], set()).add((one["kernel"], numbers(one["symbol"])[3:], len(got["launches"])))
    for t in (0, 2):
        few = {v for k, v, _ in products[t] if k == "f8_product_few_kernel"}
        assert few == {(m, *rest) for m in (1, 2) for rest in ((4, 1, 1), (1, 2, 4), (1, 2, 8))}, t
        assert {(v, parts) for k, v, parts in products[t] if k == "f8_product_tile_kernel"} == {(tile, parts) for tile in ((4, 2, 2, 4), (2, 2, 2, 2)) for parts in (1, 2)}, t
