"""What the MXFP4 entry points launch for row counts up to the largest that they accept, without a GPU: the HIP runtime's entry
points are taken by a stand-in that hands every launch to the test.  A launch takes fewer than 2^32 threads along an axis, and
the launches of a call together have to take every row once."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAX_ROWS = 2 ** 31 - 65536 - 1
BASE = 1 << 44                    # pointers are counted with, never followed
OUT = 1 << 45

STAND_IN = r"""
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim3_;
static void (*launched)(const void *, unsigned, unsigned, unsigned, unsigned, unsigned, unsigned, void **);
static void (*registered)(const void *, const char *);
static dim3_ grid_, block_;
static size_t lds_;
static void *stream_;
void stand_in(void *on_launch, void *on_register) { launched = on_launch, registered = on_register; }
void **__hipRegisterFatBinary(const void *d) { static void *x; return &x; }
void __hipUnregisterFatBinary(void **m) {}
void __hipRegisterFunction(void **m, const void *f, char *n, const char *name, unsigned l, void *a, void *b, void *c, void *d, int *w)
{
    registered(f, name);
}
void __hipRegisterVar(void **m, void *v, char *h, char *n, int e, size_t s, int c, int g) {}
int __hipPushCallConfiguration(dim3_ g, dim3_ b, size_t lds, void *s) { grid_ = g, block_ = b, lds_ = lds, stream_ = s; return 0; }
int __hipPopCallConfiguration(dim3_ *g, dim3_ *b, size_t *lds, void **s) { *g = grid_, *b = block_, *lds = lds_, *s = stream_; return 0; }
int hipLaunchKernel(const void *f, dim3_ g, dim3_ b, void **args, size_t lds, void *s)
{
    launched(f, g.x, g.y, g.z, b.x, b.y, b.z, args);
    return 0;
}
int hipFuncSetAttribute(const void *f, int a, int v) { return 0; }
int hipGetLastError(void) { return 0; }
"""

# In a process of its own, where nothing has loaded the real runtime's symbols into the global scope.
CALLER = r"""
import ctypes as C, json, re, sys
stand_in, library, calls = sys.argv[1], sys.argv[2], json.loads(sys.argv[3])
S = C.CDLL(stand_in, mode=C.RTLD_GLOBAL)
names, made = {}, []
def value(args, i, t):
    return C.cast(args[i], C.POINTER(t))[0]
class Table(C.Structure):
    _fields_ = [("codes", C.c_uint64), ("scales", C.c_uint64), ("norms", C.c_uint64), ("n", C.c_int), ("nb", C.c_int), ("sp", C.c_int)]
def on_launch(f, gx, gy, gz, bx, by, bz, args):
    name = re.search(r"\d+([a-z_]+_kernel)", names[f].decode()).group(1)
    one = dict(kernel=name, grid=[gx, gy, gz], block=[bx, by, bz])
    if name == "quantise_kernel":
        one.update(x=value(args, 0, C.c_uint64), n=value(args, 1, C.c_int64), group=value(args, 4, C.c_int),
                   codes=value(args, 7, C.c_uint64), scales=value(args, 8, C.c_uint64), norms=value(args, 9, C.c_uint64))
    elif name == "rows_kernel":
        t = value(args, 0, Table)
        one.update(codes=t.codes, scales=t.scales, table_n=t.n, ids=value(args, 2, C.c_uint64), n=value(args, 3, C.c_int64),
                   group=value(args, 4, C.c_int), out=value(args, 6, C.c_uint64))
    made.append(one)
launch_t = C.CFUNCTYPE(None, C.c_void_p, *[C.c_uint] * 6, C.POINTER(C.c_void_p))
register_t = C.CFUNCTYPE(None, C.c_void_p, C.c_char_p)
on_launch, on_register = launch_t(on_launch), register_t(lambda f, name: names.__setitem__(f, name))
S.stand_in(on_launch, on_register)
L = C.CDLL(library)
vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
L.efanna_mx_quantise.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, vp]
L.efanna_mx_rows.argtypes = [vp, vp, i64, i32, vp, i64, C.c_float, i32, vp, vp]
L.efanna_mx_product.argtypes = [vp, vp, i64, vp, vp, i64, i32, i32, vp, i64, vp]
L.efanna_mx_nearest_workspace_bytes.restype = sz
L.efanna_mx_nearest_workspace_bytes.argtypes = [i64, i32, i64, i32]
L.efanna_mx_nearest.argtypes = [vp, vp, vp, i64, i32, vp, vp, vp, i64, i32, i64, vp, vp, vp, sz, vp]
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
        return answers
    return run


COUNTS = [1, 1000, 2 ** 26, 2 ** 26 + 1, 2 ** 27 + 5, 2 ** 30 + 3, MAX_ROWS]


@pytest.mark.parametrize("d,group", [(1, 4), (32, 4), (50, 8), (128, 16), (200, 32), (257, 64), (1024, 64), (65536, 64)])
def test_quantise_takes_every_row_once(launches, d, group):
    nb = (d + 31) // 32
    sp = (nb + 3) // 4 * 4
    ldx = d + 3
    for n, got in zip(COUNTS, launches([("efanna_mx_quantise", (BASE, 2, n, d, ldx, 2 * BASE, 3 * BASE, 4 * BASE, None))
                                        for n in COUNTS])):
        assert got["status"] == 0
        done = 0
        for one in got["launches"]:
            assert one["kernel"] == "quantise_kernel" and one["block"] == [256, 1, 1] and one["group"] == group
            assert one["x"] == BASE + done * ldx * 2 and one["codes"] == 2 * BASE + done * nb * 16
            assert one["scales"] == 3 * BASE + done * sp and one["norms"] == 4 * BASE + done * 4
            assert one["grid"] == [-(-one["n"] // (256 // group)), 1, 1]
            done += one["n"]
        assert done == n


@pytest.mark.parametrize("ids", [None, 5 * BASE])
@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
@pytest.mark.parametrize("d", [1, 50, 300, 65536])
def test_rows_takes_every_row_once(launches, ids, dtype, size, d):
    nb = (d + 31) // 32
    sp = (nb + 3) // 4 * 4
    counts = COUNTS + [2 ** 28, 2 ** 28 + 1]
    n = MAX_ROWS
    for m, got in zip(counts, launches([("efanna_mx_rows", (BASE, 2 * BASE, n, d, ids, m, 1.0, dtype, OUT, None))
                                        for m in counts])):
        assert got["status"] == 0
        done = 0
        for one in got["launches"]:
            assert one["kernel"] == "rows_kernel" and one["block"] == [256, 1, 1]
            first = 0 if ids else done                      # row 0 of the table that the kernel is given
            assert one["codes"] == BASE + first * nb * 16 and one["scales"] == 2 * BASE + first * sp
            assert one["table_n"] == n - first
            assert one["ids"] == (ids + done * 4 if ids else 0)
            assert one["out"] == OUT + done * d * size
            assert one["grid"] == [-(-one["n"] // (4 * (256 // one["group"]))), 1, 1]
            done += one["n"]
        assert done == m


def test_queries_of_an_empty_table(launches):
    """As many as there are, each answered once: there is only the choice to launch, a wave for each query."""
    for nq, got in zip(COUNTS, launches([("efanna_mx_nearest", (None, None, None, 0, 64, BASE, BASE, BASE, nq, 3, -1, BASE, BASE,
                                                                BASE, 1 << 40, None)) for nq in COUNTS])):
        assert got["status"] == 0
        assert {one["kernel"] for one in got["launches"]} == {"pick_kernel"}
        took = sum(one["grid"][0] for one in got["launches"])
        assert nq <= took < nq + 128 * len(got["launches"])


@pytest.mark.parametrize("n,nq,k", [(1, 2 ** 27, 1), (300, 2 ** 26, 10), (MAX_ROWS, 1, 1), (MAX_ROWS, 300, 128), (MAX_ROWS, 20, 1),
                                    (20_000_000, 4096, 10)])
@pytest.mark.parametrize("d", [32, 960, 2000])
def test_nearest_of_many(launches, n, nq, k, d):
    got, = launches([("efanna_mx_nearest", (BASE, BASE, BASE, n, d, BASE, BASE, BASE, nq, k, -1, BASE, BASE, BASE, 1 << 40, None))])
    assert got["status"] == 0 and got["launches"]


@pytest.mark.parametrize("m,n,d,status", [(MAX_ROWS, 1, 64, 0), (1, MAX_ROWS, 64, 0), (32, MAX_ROWS, 500, 0), (33, MAX_ROWS, 64, 0),
                                          (2 ** 20, 2 ** 18, 64, 0), (2 ** 20, 2 ** 20, 64, -6), (2 ** 26, 2 ** 26, 64, -6),
                                          (32, 2 ** 30 + 64, 8192, -6)])
def test_products_are_launched_or_refused(launches, m, n, d, status):
    """Refused (EFANNA_EUNSUPPORTED) is only what would need terabytes."""
    got, = launches([("efanna_mx_product", (BASE, BASE, m, BASE, BASE, n, d, 2, OUT, n, None))])
    assert got["status"] == status
    assert len(got["launches"]) == (1 if status == 0 else 0)
    if status:
        assert n * d // 2 + m * n * 2 > 10 ** 12
